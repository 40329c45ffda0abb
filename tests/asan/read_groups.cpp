// The work-groups of a read of the paged cache over the grid that is launched: every piece of
// every wanted half once, nothing else, whatever the last row of the grid holds too many.  Exit
// status 0 when every check holds.
#include <stdio.h>

#include "../../paper_2608_10519_amd/csrc/paged.h"

using namespace sparstar;

static int failures = 0;

// A read of n pieces of each wanted half.
static void walk(int64_t n, bool k, bool v) {
  const int64_t wanted = n * (int(k) + int(v));
  const dim3 grid = rows_of_groups(wanted);
  const int64_t groups = int64_t(grid.x) * grid.y;
  bool good = groups >= wanted && grid.x <= 1u << 20;
  int64_t done[2] = {0, 0};  // pieces of K and V so far, in order
  for (int64_t w = 0; w < groups; ++w) {
    const ReadGroup r = read_group(w, n, k, v);
    if (!r.any) continue;
    good = good && (r.is_v ? v : k) && r.at == done[r.is_v]++;
  }
  good = good && done[0] == (k ? n : 0) && done[1] == (v ? n : 0);
  printf("%lld groups, k %d, v %d, grid %u x %u: %s\n", (long long)n, k, v, grid.x, grid.y, good ? "ok" : "WRONG");
  failures += !good;
}

int main() {
  const int64_t row = 1 << 20;
  // (the last: 8 x 64 heads of 144,512 rows at D = 128)
  for (const int64_t n : {int64_t(1), int64_t(7), row - 1, row, row + 1, 2 * row - 1, 2 * row + 1, 3 * row + 5, int64_t(2312192)})
    for (int want = 1; want < 4; ++want) walk(n, want & 1, want & 2);
  return failures != 0;
}
