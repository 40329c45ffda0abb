// How an attention call over the paged cache is cut up (host code).
#pragma once

#include "cache_plan.h"

namespace sparstar {

// As for the 8-bit cache (waves == 1: the kernels for up to 32 rows).
using PagedPlan = CachePlan;

constexpr int kPagedMaxRanges = 64;  // of a call of up to 32 rows

// The most ranges that a call of up to 32 rows is cut into, whatever its lists hold.
inline int paged_token_most_ranges(int64_t bh, int64_t lk, int block) {
  const int64_t nk = (lk + block - 1) / block;
  return (int)std::max<int64_t>(1, std::min<int64_t>({512 / bh, nk, kPagedMaxRanges}));
}

inline PagedPlan paged_attn_plan(int64_t bh, int64_t lq, int64_t lk, int d, int block, int64_t kv_stride, bool dense,
                                 bool may_split) {
  if (lq > 32) return cache_attn_plan(bh, lq, lk, d, block, kv_stride, dense, may_split);
  const int64_t nk = (lk + block - 1) / block, tiles = (dense ? nk : std::min(nk, kv_stride)) * (block / 64);
  PagedPlan p{1, 1, 0, 0, 0};
  if (may_split && tiles >= 12 * kTokenWaves)
    p.ranges = (int)std::min<int64_t>(paged_token_most_ranges(bh, lk, block), tiles / (4 * kTokenWaves));
  p.grid = bh * p.ranges;
  return p;
}

// Bytes of workspace: the ranges' results, fp32 for up to 32 rows, and four values per row.
inline size_t paged_part_bytes(int64_t rows, int64_t lq, int d, int ranges) {
  return lq > 32 ? cache_part_o_bytes(rows, d, ranges) : (size_t(rows * d) * ranges * 4 + 255) & ~size_t(255);
}
inline size_t paged_attn_workspace(int64_t bh, int64_t lq, int64_t lk, int d, int block) {
  const int ranges = lq > 32 ? cache_attn_most_ranges(bh, lq, lk, block) : paged_token_most_ranges(bh, lk, block);
  return ranges > 1 ? paged_part_bytes(bh * lq, lq, d, ranges) + size_t(bh * lq) * ranges * 4 * sizeof(float) : 0;
}

// Threads of the largest launch of a call, of which there may be fewer than 2^32.
inline int64_t paged_attn_threads(const PagedPlan& p, int64_t rows, int d) {
  if (p.waves > 1) return cache_attn_threads(p, rows, d);
  return std::max<int64_t>(p.grid * 64 * kTokenWaves, p.ranges > 1 ? rows * d * 4 : 0);
}

}  // namespace sparstar
