// The host side of the gradient and cache calls under the address and
// undefined-behaviour sanitizers.  The launchers here fail, after checking that
// what the call hands the kernels lies inside the workspace it asked for.  Fake
// device pointers are never dereferenced.  Exit status 0 when every check holds.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <random>

#include "../../include/sparstar.h"
#include "../../paper_2608_10519_amd/csrc/bwd_plan.h"
#include "../../paper_2608_10519_amd/csrc/cache_plan.h"

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

static char* const F = (char*)0x10000;  // 256-byte aligned, never dereferenced
static char* const W = (char*)(uintptr_t(1) << 50);  // the workspace, and its size
static size_t ws_bytes = 0;

// [p, p + n) inside the workspace
static bool inside(const void* p, double n) {
  const double at = double(static_cast<const char*>(p) - W);
  return at >= 0 && at + n <= double(ws_bytes);
}

namespace sparstar {

hipError_t launch_cache_write(const CacheWriteArgs& a, int, int block, hipStream_t) {
  ++launches;
  const int64_t blocks = (a.cap + block - 1) / block;
  // with the rows known, the last block that a work-group takes is one of the cache's
  if (a.starts == nullptr) CHECK(a.start / block + a.n_blocks <= blocks);
  CHECK(int64_t(a.n_blocks) * block >= a.l);
  return hipErrorInvalidValue;
}
hipError_t launch_cache_read(const CacheReadArgs& a, hipStream_t) {
  ++launches;
  CHECK(a.start >= 0 && a.start + a.l <= a.cap);
  return hipErrorInvalidValue;
}
hipError_t launch_cache_attn(const CacheAttnArgs& a, int d, int waves, bool dense, hipStream_t) {
  ++launches;
  const double rows = double(a.bh) * a.lq;
  CHECK(a.ranges >= 1 && (a.ranges == 1 || (inside(a.part_o, 2.0 * rows * d * a.ranges) &&
                                            inside(a.part_meta, 16.0 * rows * a.ranges) &&
                                            (char*)a.part_o + size_t(2.0 * rows * d * a.ranges) <= (char*)a.part_meta)));
  CHECK((a.lq <= 32) == (waves == 1));
  CHECK(waves == 1 || waves == 2 || waves == 4);
  if (!dense && waves > 1) CHECK(waves * 32 == a.block);
  const int64_t groups = a.lq <= 32 ? 1 : (a.lq + 32 * waves - 1) / (32 * waves);
  CHECK(a.grid >= int64_t(a.bh) * a.ranges * groups);
  return hipErrorInvalidValue;
}
hipError_t launch_attn_bwd(const BwdArgs& a, int d, bool dense, hipStream_t) {
  ++launches;
  const double lq = double(a.lq), lk = double(a.lk);
  CHECK(inside(a.stats, double(a.bh) * a.n_q * a.block * 8));
  if (!dense) CHECK(inside(a.bits, 4.0 * a.bh * a.n_k * a.n_words));
  if (!dense) CHECK((char*)a.stats + size_t(double(a.bh) * a.n_q * a.block * 8) <= (char*)a.bits);
  CHECK(a.dq_ranges >= 1 && a.dkv_ranges >= 1);
  if (a.list_min > 0) {
    // The lists hold `entries` at most.  A block with c > piece_max of them is cut into ceil(c / piece_max) < 2 c /
    // piece_max pieces, at most c / piece_max beyond the first; one with c > list_min is taken whole.
    const double entries = double(a.bh) * a.n_q * std::min(a.stride, a.n_k), blocks = double(a.bh) * a.n_k;
    const bool cut = a.n_q > a.piece_max;
    const double pieces =
        cut ? std::min(2 * entries / a.piece_max, blocks * ((a.n_q + a.piece_max - 1) / a.piece_max)) : 0;
    const double extra = cut ? std::min(entries / a.piece_max, pieces) : 0;
    const double whole = a.list_min < a.piece_max ? floor(entries / (a.list_min + 1)) : 0;
    CHECK(!dense && a.dkv_ranges == 1 && a.piece_max >= a.list_min && pieces + whole <= a.most_pieces);
    CHECK((char*)a.bits + size_t(4.0 * a.bh * a.n_k * a.n_words) <= (char*)a.piece_count);
    CHECK((char*)(a.piece_count + 2) <= (char*)a.pieces && reinterpret_cast<uintptr_t>(a.pieces) % 16 == 0);
    CHECK((char*)a.pieces + size_t(16.0 * (blocks + extra)) <= (char*)a.listed);
    CHECK((char*)a.listed + size_t(blocks) <= (char*)a.part);
    CHECK((char*)a.part_kv <= (char*)a.part_piece);
    CHECK(inside(a.part_piece, 8.0 * pieces * a.block * d));
  }
  if (a.dq_ranges > 1) CHECK(inside(a.part, 4.0 * a.bh * lq * d * a.dq_ranges));
  if (a.dkv_ranges > 1) CHECK(inside(a.part_kv, 8.0 * a.bh * lk * d * a.dkv_ranges));
  // (the two may be in use at the same time)
  if (a.dq_ranges > 1) CHECK((char*)a.part + size_t(4.0 * a.bh * lq * d * a.dq_ranges) <= (char*)a.part_kv);
  CHECK(isfinite(a.scale) && isfinite(a.inv_scale) && isfinite(a.scale_log2));
  return hipErrorInvalidValue;
}

}  // namespace sparstar

int main() {
  std::mt19937_64 rng(7);
  auto pick = [&](int64_t lo, int64_t hi) { return lo + int64_t(rng() % uint64_t(hi - lo + 1)); };
  // lengths and head counts over their orders of magnitude
  auto size = [&](int64_t most) { return std::min<int64_t>(most, std::max<int64_t>(1, int64_t(exp2(pick(0, 2000) / 100.0)))); };
  float* const f = (float*)F;
  uint8_t* const u = (uint8_t*)F;
  int32_t* const n = (int32_t*)F;
  for (int i = 0; i < 4000; ++i) {
    const int B = int(pick(1, 3)), H = int(pick(1, 40)), D = pick(0, 1) ? 64 : 128, b = pick(0, 1) ? 64 : 128;
    const int64_t Lq = pick(0, 9) == 0 ? pick(0, 33) : size(200000), Lk = size(1 << 20), cap = Lk + pick(0, 300);
    const int stride = int(pick(1, (Lk + b - 1) / b + 3));
    ws_bytes = sparstar_attn_bwd_workspace_bytes(B, H, Lq, Lk, D, b);
    launches = 0;
    int rc = sparstar_sparse_attn_bwd(F, F, F, F, f, F, i % 2 ? f : nullptr, B, H, Lq, Lk, D, b, n, n, stride, 0.f, F,
                                      F, F, W, ws_bytes, nullptr);
    CHECK(rc == SPARSTAR_ERR_HIP);
    rc = sparstar_dense_attn_bwd(F, F, F, F, f, F, nullptr, B, H, Lq, Lk, D, b, 0.3f, F, F, F, W, ws_bytes, nullptr);
    CHECK(rc == SPARSTAR_ERR_HIP && launches == 2);

    ws_bytes = sparstar_cache_attn_workspace_bytes(B, H, Lq, Lk, D, b);
    launches = 0;
    void* const ws = i % 3 ? W : nullptr;
    rc = sparstar_cache_sparse_attn_fwd(F, F, F, u, u, B, H, Lq, Lk, cap, D, b, nullptr, n, n, stride, 0.f, F, f, ws,
                                        ws ? ws_bytes : 0, nullptr);
    CHECK(rc == (Lq == 0 ? SPARSTAR_OK : SPARSTAR_ERR_HIP));
    rc = sparstar_cache_dense_attn_fwd(F, F, F, u, u, B, H, Lq, Lk, cap, D, b, n, 0.f, F, nullptr, ws,
                                       ws ? ws_bytes : 0, nullptr);
    CHECK(rc == (Lq == 0 ? SPARSTAR_OK : SPARSTAR_ERR_HIP));
    CHECK(launches == (Lq == 0 ? 0 : 2));

    const int64_t start = pick(0, cap), L = pick(0, cap - start);
    launches = 0;
    rc = sparstar_cache_write(F, F, B, H, L, D, b, start, i % 5 ? nullptr : n, nullptr, cap, F, F, u, u, nullptr);
    CHECK(rc == (L == 0 ? SPARSTAR_OK : SPARSTAR_ERR_HIP));
    rc = sparstar_cache_read(F, F, u, u, B, H, start, L, cap, D, b, i % 2 ? F : nullptr, F, nullptr);
    CHECK(rc == (L == 0 ? SPARSTAR_OK : SPARSTAR_ERR_HIP) && launches == (L == 0 ? 0 : 2));
  }
  // refusals write a message and launch nothing
  launches = 0;
  ws_bytes = size_t(1) << 40;
  CHECK(sparstar_dense_attn_bwd(F, F, F, F, f, F, nullptr, 1, 1, 64, 64, 64, 64, NAN, F, F, F, W, ws_bytes, nullptr) ==
        SPARSTAR_ERR_INVALID_ARG);
  CHECK(strstr(sparstar_last_error(), "finite") != nullptr);
  CHECK(sparstar_dense_attn_bwd(F, F, F, F, f, F, nullptr, 1, 1, 64, 64, 64, 64, 0.f, F, F, F, W, 0, nullptr) ==
        SPARSTAR_ERR_WORKSPACE);
  CHECK(sparstar_cache_write(F, F, 1, 1, 5, 64, 64, INT64_MAX, nullptr, nullptr, 64, F, F, u, u, nullptr) ==
        SPARSTAR_ERR_INVALID_ARG);
  CHECK(sparstar_cache_write(F, F, 1, 1, 5, 64, 64, -1, nullptr, nullptr, 64, F, F, u, u, nullptr) ==
        SPARSTAR_ERR_INVALID_ARG);
  CHECK(sparstar_cache_read(F, F, u, u, 1, 1, INT64_MIN, 5, 64, 64, 64, F, F, nullptr) == SPARSTAR_ERR_INVALID_ARG);
  CHECK(sparstar_cache_read(F, F, u, u, 1, 1, 0, INT64_MAX, 64, 64, 64, F, F, nullptr) == SPARSTAR_ERR_INVALID_ARG);
  CHECK(sparstar_cache_dense_attn_fwd(F, F, F, u, u, 1, 1, 64, INT64_MAX, 64, 64, 64, nullptr, 0.f, F, f, nullptr, 0,
                                      nullptr) == SPARSTAR_ERR_INVALID_ARG);
  CHECK(launches == 0);
  printf("%d checks passed, %d failed\n", passes, failures);
  return failures != 0;
}
