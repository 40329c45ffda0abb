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

// The same of more rows: the 8-bit cache's, and beyond its 16 as many as fill the chip four times
// with a wave per 32 rows, of two blocks at least.
inline int paged_rows_most_ranges(int64_t bh, int64_t lq, int64_t lk, int block) {
  const int64_t nk = (lk + block - 1) / block, waves = bh * ((lq + 31) / 32);
  const int base = cache_attn_most_ranges(bh, lq, lk, block);
  return base < kSplits ? base : (int)std::max<int64_t>(base, std::min<int64_t>({4096 / std::max<int64_t>(waves, 1), nk / 2, 64}));
}

// More than 32 rows take the 8-bit cache's cut, whose ranges are a power of two, or such a number
// of ranges that their work-groups fill the chip once, twice or three times and leave nothing
// over, where the estimate finds that faster by 2% (calls of more than 200 us in few rounds: any number).  24
// heads of 128 x 144,512 340 us in 16 ranges, 276 in 21; 18 of 220 x 10,061 59 us in 8, 44 in 14;
// 24 of 64 x 144,512 187 us in 32, 175 in 42.
inline CachePlan paged_rows_plan(int64_t bh, int64_t lq, int64_t lk, int d, int block, int64_t kv_stride, bool dense,
                                 bool may_split) {
  CachePlan p = cache_attn_plan(bh, lq, lk, d, block, kv_stride, dense, may_split);
  if (p.ranges == 1 && !may_split) return p;
  const int64_t nk = (lk + block - 1) / block;
  const int most = paged_rows_most_ranges(bh, lq, lk, block);
  const bool full = dense || kv_stride >= nk;
  const double rho = full ? 1.0 : double(kv_stride) / double(nk);
  auto time = [&](int ranges, int rows) {
    return attn_time_us(bh, lq, lk, d, block, rho, full, ranges, p.rotation > 0, rows);
  };
  double best = 0.98 * time(p.ranges, 32 * p.waves);
  int ranges = p.ranges, rows = 32 * p.waves;
  for (int w = dense ? 64 : block; w <= (dense ? 128 : block); w *= 2) {
    const int64_t items = bh * ((lq + w - 1) / w), held = 256 * 4 * kAttnWavesPerSimd * 32 / w;
    const bool any = best > 200.0 && items <= 4 * held;
    for (int i = 1; i <= (any ? most : 3); ++i) {
      const int64_t r = any ? i : i * held / items;
      if (r < 2 || r > most || nk < r) continue;
      if (attn_grid(bh * r, (lq + w - 1) / w, 0) * 2 * w >> 32) break;  // launch limit
      if (const double t = time(int(r), w); t < best) best = t, ranges = int(r), rows = w;
    }
  }
  p.waves = rows / 32;
  p.ranges = ranges;
  const int64_t groups = (lq + rows - 1) / rows;
  p.spread_bits = attn_spread_bits(bh * ranges, groups, rows);
  p.grid = attn_grid(bh * ranges, groups, p.spread_bits);
  if (p.rotation > 0) p.rotation = 32 * 4 * kAttnWavesPerSimd / p.waves;
  return p;
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
  if (lq > 32) return PagedPlan{paged_rows_plan(bh, lq, lk, d, block, kv_stride, dense, may_split), 0};
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
  const int ranges = lq > 32 ? paged_rows_most_ranges(bh, lq, lk, block) : paged_token_most_ranges(bh, lk, block);
  return ranges > 1 ? paged_part_bytes(bh * lq, lq, d, ranges) + size_t(bh * lq) * ranges * 4 * sizeof(float) : 0;
}

// Threads of the largest launch of a call, of which there may be fewer than 2^32.
inline int64_t paged_attn_threads(const PagedPlan& p, int64_t rows, int d) {
  if (p.waves > 1) return cache_attn_threads(p, rows, d);
  return std::max<int64_t>(p.grid * 64 * p.token_waves, p.ranges > 1 ? rows * d * 4 : 0);
}

}  // namespace sparstar
