// The host side of the rotary and paged-cache calls under the address and
// undefined-behaviour sanitizers.  The launchers here fail, after checking that what the
// call hands the kernels is consistent and lies inside the workspace it asked for.  Fake
// device pointers are never dereferenced.  Exit status 0 when every check holds.
#include <limits.h>
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <random>

#include "../../include/sparstar.h"
#include "../../paper_2608_10519_amd/csrc/paged.h"
#include "../../paper_2608_10519_amd/csrc/paged_plan.h"

static int failures = 0, passes = 0, launches = 0;

#define CHECK(cond)                                           \
  do {                                                        \
    if (!(cond)) {                                            \
      fprintf(stderr, "FAIL line %d: %s\n", __LINE__, #cond); \
      ++failures;                                             \
    } else {                                                  \
      ++passes;                                               \
    }                                                         \
  } while (0)

static char* const F = (char*)0x10000;               // 256-byte aligned, never dereferenced
static char* const W = (char*)(uintptr_t(1) << 50);  // the workspace, and its size
static size_t ws_bytes = 0;

static bool inside(const void* p, double n) {
  const double at = double(static_cast<const char*>(p) - W);
  return at >= 0 && at + n <= double(ws_bytes);
}

namespace sparstar {

hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t) {
  ++launches;
  for (int p = 0; p < a.pairs; ++p) {
    CHECK(a.axis[p] < a.axes);
    // quarter turns of the furthest coordinate fit the kernel's rounding
    CHECK(fabs(a.quarters[p]) * 2147483648.0 < double(int64_t(1) << 51));
  }
  return hipErrorInvalidValue;
}
hipError_t launch_rope(const RopeArgs& a, hipStream_t) {
  ++launches;
  CHECK(a.turn.pairs % 8 == 0 && 2 * a.turn.pairs <= a.d);
  CHECK(a.turn.positions != nullptr || (a.start >= 0 && a.start + a.l <= a.turn.table_rows));
  CHECK(a.xs.b % 8 == 0 && a.xs.h % 8 == 0 && a.xs.l % 8 == 0 && a.xs.b >= 0 && a.xs.h >= 0 && a.xs.l >= 0);
  return hipErrorInvalidValue;
}
hipError_t launch_paged_write(const PagedArgs& a, hipStream_t) {
  ++launches;
  CHECK(a.starts != nullptr || (a.start >= 0 && a.start + a.l <= a.n_table * a.block));
  CHECK(a.turn.table == nullptr || a.turn.positions != nullptr || a.starts != nullptr ||
        a.start + a.l <= a.turn.table_rows);
  return hipErrorInvalidValue;
}
hipError_t launch_paged_read(const PagedArgs& a, hipStream_t) {
  ++launches;
  CHECK(a.start >= 0 && a.start + a.l <= a.n_table * a.block && (a.k_out || a.v_out));
  return hipErrorInvalidValue;
}
hipError_t launch_paged_attn(const PagedAttnArgs& a, int d, bool dense, hipStream_t) {
  ++launches;
  const double rows = double(a.bh) * a.lq;
  CHECK((a.lq <= 32) == (a.waves == 1));
  CHECK(a.lk <= a.n_table * a.block);
  if (a.waves == 1) {
    CHECK(a.token_waves == 4 || a.token_waves == 8);
    CHECK(a.ranges >= 1 && a.ranges <= kPagedMaxRanges && a.grid == int64_t(a.bh) * a.ranges);
    if (a.ranges > 1)
      CHECK(inside(a.part32, 4.0 * rows * d * a.ranges) && inside(a.part_meta, 16.0 * rows * a.ranges) &&
            (char*)a.part32 + size_t(4.0 * rows * d * a.ranges) <= (char*)a.part_meta);
  } else {
    CHECK(a.waves == 2 || a.waves == 4);
    if (!dense) CHECK(a.waves * 32 == a.block);
    const int64_t groups = (a.lq + 32 * a.waves - 1) / (32 * a.waves);
    CHECK(a.grid >= int64_t(a.bh) * a.ranges * groups && a.grid * 64 * a.waves < int64_t(1) << 32);
    CHECK(a.spread_bits >= 0 && a.spread_bits <= 3);
    // every item has a work-group that finds it (the kernel's decode of blockIdx)
    const int64_t pairs = int64_t(a.bh) * a.ranges, bits = a.spread_bits;
    if (bits < 3) CHECK((pairs << bits) % 8 == 0 && a.grid == (pairs << bits) * ((groups + (1 << bits) - 1) >> bits));
    else CHECK(a.grid == pairs * groups);
    if (a.ranges > 1)
      CHECK(inside(a.part_o, 2.0 * rows * d * a.ranges) && inside(a.part_meta, 16.0 * rows * a.ranges) &&
            (char*)a.part_o + size_t(2.0 * rows * d * a.ranges) <= (char*)a.part_meta);
  }
  return hipErrorInvalidValue;
}

}  // namespace sparstar

int main() {
  std::mt19937_64 rng(11);
  auto pick = [&](int64_t lo, int64_t hi) { return lo + int64_t(rng() % uint64_t(hi - lo + 1)); };
  // lengths and head counts over their orders of magnitude
  auto size = [&](int64_t most) { return std::min<int64_t>(most, std::max<int64_t>(1, int64_t(exp2(pick(0, 2000) / 100.0)))); };
  float* const f = (float*)F;
  uint8_t* const u = (uint8_t*)F;
  int32_t* const n = (int32_t*)F;
  for (int i = 0; i < 4000; ++i) {
    const int B = int(pick(1, 3)), H = int(pick(1, 40)), D = pick(0, 1) ? 64 : 128, b = pick(0, 1) ? 64 : 128;
    const int64_t Lq = pick(0, 9) == 0 ? pick(0, 33) : size(200000), Lk = size(1 << 20), nt = (Lk + b - 1) / b + pick(0, 3);
    const int stride = int(pick(1, (Lk + b - 1) / b + 3)), pairs = int(8 * pick(1, D / 16));
    ws_bytes = sparstar_paged_attn_workspace_bytes(B, H, Lq, Lk, D, b);
    launches = 0;
    void* const ws = i % 3 ? W : nullptr;
    int rc = sparstar_paged_sparse_attn_fwd(F, F, F, u, u, B, H, Lq, Lk, D, b, n, nt, 100, nullptr, n, n, stride, 0.f, F, f,
                                            ws, ws ? ws_bytes : 0, nullptr);
    CHECK(rc == (Lq == 0 ? SPARSTAR_OK : SPARSTAR_ERR_HIP));
    rc = sparstar_paged_dense_attn_fwd(F, F, F, u, u, B, H, Lq, Lk, D, b, n, nt, 100, n, 0.f, F, nullptr, ws,
                                       ws ? ws_bytes : 0, nullptr);
    CHECK(rc == (Lq == 0 ? SPARSTAR_OK : SPARSTAR_ERR_HIP));
    CHECK(launches == (Lq == 0 ? 0 : 2));

    const int64_t start = pick(0, nt * b), L = pick(0, nt * b - start);
    const sparstar_strides dense{H * L * D, L * D, D}, packed{3 * L * H * D, D, 3 * int64_t(H) * D};
    const sparstar_strides s = i % 2 ? dense : packed;
    launches = 0;
    rc = sparstar_paged_write(F, s, F, dense, B, H, L, D, b, start, i % 5 ? nullptr : n, nullptr, i % 4 ? f : nullptr,
                              start + L + (start + L == 0), pairs, i % 3 == 0, nullptr, n, nt, 100, F, F, u, u, nullptr);
    CHECK(rc == (L == 0 ? SPARSTAR_OK : SPARSTAR_ERR_HIP));
    rc = sparstar_paged_read(F, F, u, u, B, H, start, L, D, b, n, nt, 100, i % 2 ? F : nullptr, F, nullptr);
    CHECK(rc == (L == 0 ? SPARSTAR_OK : SPARSTAR_ERR_HIP));
    rc = sparstar_rope_fwd(F, s, B, H, L, D, f, 7 + L, pairs, i % 2, nullptr, 7, F + (int64_t(1) << 40), packed, nullptr);
    CHECK(rc == (L == 0 ? SPARSTAR_OK : SPARSTAR_ERR_HIP));
    rc = sparstar_rope_bwd(F, s, B, H, L, D, f, 1, pairs, i % 2, n, 0, F, s, nullptr);
    CHECK(rc == (L == 0 ? SPARSTAR_OK : SPARSTAR_ERR_HIP));
    CHECK(launches == (L == 0 ? 0 : 4));
    double freq[64];
    int32_t axis[64];
    for (int p = 0; p < 64; ++p) freq[p] = (p % 2 ? -1 : 1) * 1048576.0 / (1 + p), axis[p] = p % 3;
    CHECK(sparstar_rope_table(n, size(1 << 20), 3, int(pick(1, 64)), freq, axis, 1.0, f, nullptr) == SPARSTAR_ERR_HIP);
  }
  // refusals write a message and launch nothing
  launches = 0;
  const sparstar_strides big{INT64_MAX - 7, INT64_MAX - 7, INT64_MAX - 7}, low{INT64_MIN, 0, 0}, one{0, 0, 64};
  for (const sparstar_strides& s : {big, low}) {
    CHECK(sparstar_rope_fwd(F, s, 2, 2, 2, 64, f, 9, 32, 0, nullptr, 0, F, one, nullptr) == SPARSTAR_ERR_INVALID_ARG);
    CHECK(sparstar_paged_write(F, one, F, s, 2, 2, 2, 64, 64, 0, nullptr, nullptr, nullptr, 0, 0, 0, nullptr, n, 1, 1, F,
                               F, u, u, nullptr) == SPARSTAR_ERR_INVALID_ARG);
    CHECK(strstr(sparstar_last_error(), "v: ") != nullptr);
  }
  for (int64_t start : {INT64_MIN, int64_t(-1), INT64_MAX}) {
    CHECK(sparstar_rope_fwd(F, one, 1, 1, 2, 64, f, 9, 32, 0, nullptr, start, F, one, nullptr) == SPARSTAR_ERR_INVALID_ARG);
    CHECK(sparstar_paged_write(F, one, F, one, 1, 1, 2, 64, 64, start, nullptr, nullptr, nullptr, 0, 0, 0, nullptr, n, 1,
                               1, F, F, u, u, nullptr) == SPARSTAR_ERR_INVALID_ARG);
    CHECK(sparstar_paged_read(F, F, u, u, 1, 1, start, 2, 64, 64, n, 1, 1, F, F, nullptr) == SPARSTAR_ERR_INVALID_ARG);
  }
  for (int64_t x : {INT64_MIN, int64_t(0), INT64_MAX}) {
    CHECK(sparstar_paged_dense_attn_fwd(F, F, F, u, u, 1, 1, 2, 64, 64, 64, n, x, 9, nullptr, 0.f, F, f, nullptr, 0,
                                        nullptr) == SPARSTAR_ERR_INVALID_ARG);
    CHECK(sparstar_paged_dense_attn_fwd(F, F, F, u, u, 1, 1, 2, 64, 64, 64, n, 9, x, nullptr, 0.f, F, f, nullptr, 0,
                                        nullptr) == SPARSTAR_ERR_INVALID_ARG);
    if (x != 0) CHECK(sparstar_rope_table(n, x, 1, 4, (const double[4]){1, 1, 1, 1}, nullptr, 1.0, f, nullptr) ==
                      SPARSTAR_ERR_INVALID_ARG);
  }
  CHECK(launches == 0);
  printf("%d checks passed, %d failed\n", passes, failures);
  return failures != 0;
}
