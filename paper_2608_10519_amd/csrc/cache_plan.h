// How an attention call over the 8-bit cache is cut up (host code): waves per
// work-group, ranges of each list, and the order of the work-groups.  The kernels
// (cache_attn.hip) take the cut through CacheAttnArgs.
#pragma once

#include <algorithm>

#include "attn_plan.h"

namespace sparstar {

struct CachePlan {
  int waves;        // of a work-group, 32 query rows each
  int ranges;       // of each list's entries
  int rotation;     // as in AttnPlan
  int spread_bits;
  int64_t grid;
};

constexpr int kCacheMaxTokenRanges = 64;
// For more rows the ranges are the bf16 forward's, and beyond its 16 as many as keep two waves
// per SIMD busy, of four blocks at least.  One head of 64 x 144,512: 62 us in 64 ranges, 110 in
// 32, 216 in 16; 24 heads of 64 x 84,032 132 and 191, 3 heads of 100 x 9,000 17.4 and 27.
constexpr int kCacheMaxRanges = 64;
constexpr int kCacheWaves = 2048;

// The most ranges that a call of these sizes is cut into, whatever its lists hold.
inline int cache_attn_most_ranges(int64_t bh, int64_t lq, int64_t lk, int block) {
  const int64_t nk = (lk + block - 1) / block;
  if (lq > 32) {
    int r = nk >= kSplits ? kSplits : 1;
    const int64_t waves = bh * ((lq + block - 1) / block) * (block / 32);
    while (r >= kSplits && r < kCacheMaxRanges && 2 * r * waves <= kCacheWaves && nk >= 8 * r) r *= 2;
    return r;
  }
  return (int)std::max<int64_t>(1, std::min<int64_t>({1024 / kTokenWaves / bh, nk, kCacheMaxTokenRanges}));
}

// kv_stride: entries that a list can hold; ignored for the dense call.
inline CachePlan cache_attn_plan(int64_t bh, int64_t lq, int64_t lk, int d, int block, int64_t kv_stride, bool dense,
                                 bool may_split) {
  const int64_t nk = (lk + block - 1) / block;
  if (lq <= 32) {
    // A few rows stream the cache: four waves to a CU (with more, some CUs get five or six and
    // the call waits for them: 1,792 waves 166 us, 2,560 197, 1,024 172 for two sequences of
    // 24 heads, 84,032 and 67,226 rows).  A second launch that joins ranges costs what 12 tiles
    // of a wave cost (8 heads, D = 128: 1,024 rows in one range 11.1 us, in two 15.0; 2,048 rows
    // 17.5 and 14.9).  A wave reads four tiles at least, and a row's ranges are bounded, since
    // joining them costs as much as reading them.
    const int64_t entries = dense ? nk : std::min(nk, kv_stride), tiles = entries * (block / attn_tile_keys(d));
    const int64_t most = cache_attn_most_ranges(bh, lq, lk, block);
    CachePlan p{1, 1, 0, 0, 0};
    if (may_split && tiles >= 12 * kTokenWaves)
      p.ranges = (int)std::min<int64_t>(most, tiles / (4 * kTokenWaves));
    p.grid = bh * p.ranges;
    return p;
  }
  const AttnPlan p = attn_plan(bh, lq, lk, d, block, kv_stride, dense, may_split && nk >= kSplits);
  CachePlan c{p.group_rows / 32, p.ranges, p.rotation, p.spread_bits, p.grid};
  if (c.ranges == kSplits) {
    const int64_t entries = dense ? nk : std::min(nk, kv_stride), groups = (lq + p.group_rows - 1) / p.group_rows;
    const int most = cache_attn_most_ranges(bh, lq, lk, block);
    while (c.ranges < most && entries >= 8 * c.ranges) c.ranges *= 2;
    c.spread_bits = attn_spread_bits(bh * c.ranges, groups, p.group_rows);
    c.grid = attn_grid(bh * c.ranges, groups, c.spread_bits);
  }
  return c;
}

// Groups of threads that share the join of a row's ranges (cache_merge_kernel): a group per D / 8
// threads reads a range at a time, few rows fill the chip with 16 of them.
inline int cache_join_groups(int waves, int64_t rows, int ranges) {
  return waves == 1 || rows <= 4096 || ranges > kSplits ? 16 : 1;
}

// Threads of the largest launch of a call, of which there may be fewer than 2^32.
inline int64_t cache_attn_threads(const CachePlan& p, int64_t rows, int d) {
  const int64_t join = p.ranges > 1 ? rows * (d / 8) * cache_join_groups(p.waves, rows, p.ranges) + 256 : 0;
  return std::max(p.grid * 64 * (p.waves == 1 ? kTokenWaves : p.waves), join);
}

inline size_t cache_part_o_bytes(int64_t rows, int d, int ranges) {
  return (size_t(rows * d) * ranges * 2 + 255) & ~size_t(255);
}

inline size_t cache_attn_workspace(int64_t rows, int d, int ranges) {
  return ranges > 1 ? cache_part_o_bytes(rows, d, ranges) + size_t(rows) * ranges * 4 * sizeof(float) : 0;
}

}  // namespace sparstar
