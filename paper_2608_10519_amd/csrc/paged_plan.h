// How an attention call over the paged cache is cut up (host code).
#pragma once

#include "cache_plan.h"

namespace sparstar {

// As for the 8-bit cache (waves == 1: the kernel for up to 32 rows, with token_waves waves).
struct PagedPlan : CachePlan {
  int token_waves;
};

constexpr int kPagedMaxRanges = 64;  // of a call of up to 32 rows

// The most ranges that a call of up to 32 rows is cut into, whatever its lists hold.
inline int paged_token_most_ranges(int64_t bh, int64_t lk, int block) {
  const int64_t nk = (lk + block - 1) / block;
  return (int)std::max<int64_t>(1, std::min<int64_t>({512 / bh, nk, kPagedMaxRanges}));
}

// Up to 32 rows stream the cache, in ranges of four waves each, two to a CU: more of them gain
// nothing (24 heads of 144,512 rows 92 us with 504 work-groups, 100 with 240, 94 with 768), and
// a wave reads four 64-key tiles at least.  A second launch that joins ranges costs what six
// tiles of a lone wave cost (1.1 us each at D = 128), so lists of less than 48 tiles stay whole:
// 24 heads of 4,000 rows 15.3 us in three ranges, 19.3 in one.  Where whole lists leave a CU to
// one work-group it has eight waves (24 heads of 2,048 rows 12.1 us, 13.8 with four; 64 x 24
// heads of 700 rows 51 and 36).
inline PagedPlan paged_attn_plan(int64_t bh, int64_t lq, int64_t lk, int d, int block, int64_t kv_stride, bool dense,
                                 bool may_split) {
  if (lq > 32) return PagedPlan{cache_attn_plan(bh, lq, lk, d, block, kv_stride, dense, may_split), 0};
  const int64_t nk = (lk + block - 1) / block, tiles = (dense ? nk : std::min(nk, kv_stride)) * (block / 64);
  PagedPlan p{{1, 1, 0, 0, 0}, 4};
  if (may_split && tiles >= 48) p.ranges = (int)std::min<int64_t>(paged_token_most_ranges(bh, lk, block), tiles / 16);
  if (p.ranges == 1 && tiles > 8 && bh <= 256) p.token_waves = 8;
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
  return std::max<int64_t>(p.grid * 64 * p.token_waves, p.ranges > 1 ? rows * d * 4 : 0);
}

}  // namespace sparstar
