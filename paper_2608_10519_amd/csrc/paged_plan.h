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

// The same of more rows: the 8-bit cache's, and as many as fill the chip three times with a wave
// per 32 rows, of 64 keys at least.  From 2^18 rows of all heads on no cut has more than eight
// (of 300,000 random sizes): more would only ask for a larger workspace.
inline int paged_rows_most_ranges(int64_t bh, int64_t lq, int64_t lk, int block) {
  const int64_t waves = bh * ((lq + 31) / 32), filled = 3 * 256 * 4 * kAttnWavesPerSimd / std::max<int64_t>(waves, 1);
  const int64_t most = std::max<int64_t>(cache_attn_most_ranges(bh, lq, lk, block), std::min<int64_t>({filled, (lk + 63) / 64, 64}));
  return (int)std::min<int64_t>(most, bh * lq >= 1 << 18 ? 8 : 64);
}

// The time of a call of more than 32 rows whose lists hold `keys` keys, us: its start, the tiles
// of work-groups that a CU holds one, two, three or four of (of two waves; of four: one or two),
// round after round, and the join.  (Work-groups without work take places too: the last round of
// two heads of 2,325 x 14,000, D = 64, in 13 ranges starts 8 of 520, 45 us; in 12 ranges 37.5.)  Fitted to 450
// random shapes of up to 250 us (1 to 72 heads, 33 to 6,000 x 200 to 140,000, dense and 5% to 65%,
// both head dims and block sizes), each timed at some 13 cuts, and the join's terms again, for
// results in fp32, to 300 such.  On 200 others the cut of the least estimate is 0.8% slower than
// the best one on average (the 8-bit cache's cut was 7%, up to 97%).  It ranks cuts and is no
// prediction: nine cuts in ten above 14 us take 0.83 to 1.06 times what it says, and lists
// that cluster up to a third more.
inline double paged_rows_time_us(int64_t bh, int64_t lq, int64_t keys, int d, int ranges, int rows) {
  static constexpr double kTileUs[2][2][4] = {{{.82, 1.17, 1.23, 1.32}, {.78, 1.18}}, {{.71, .95, 1.01, 1.09}, {.66, .95}}};
  static constexpr double kStart[2][2] = {{.94, 1.3}, {.64, 1.7}};  // tiles that a work-group's start costs
  const double* const us = kTileUs[d == 128][rows == 128];
  const int per_cu = 4 * kAttnWavesPerSimd * 32 / rows;
  const int64_t pairs = bh * ranges, groups = (lq + rows - 1) / rows, held = 32 * per_cu;
  const int64_t an_xcd = (attn_grid(pairs, groups, attn_spread_bits(pairs, groups, rows)) + 7) / 8;
  const int64_t whole = an_xcd / held, part = an_xcd - whole * held;
  const double tiles = double(keys) / ranges / attn_tile_keys(d) + kStart[d == 128][rows == 128];
  double t = 5.6 + double(whole) * tiles * us[per_cu - 1];
  if (part > 0) t += tiles * us[(part + 31) / 32 - 1];
  if (ranges > 1) t += 4.2 + 0.06 * ranges + double(bh) * double(lq) * ranges * (4 * d + 16) / 2.6e6;
  return t;
}

// More than 32 rows take the cut of the least estimated time, among some numbers of ranges and
// those that fill the chip once, twice or three times: 24 heads of 64 x 144,512 203 us in 32
// ranges, 173 in 42; one head of 719 x 771 22 us whole, 13.4 in 8; 50 heads of 157 rows with lists of
// 2,048 keys 53 us whole, 31 in 6.  Calls of more than 300 us, where the lists' shares of the L2
// count, take the 8-bit cache's cut, or a number of ranges that fills the chip where the forward's
// estimate finds that faster by 2%: 24 heads of 2,880 x 75,392 six ranges.
inline CachePlan paged_rows_plan(int64_t bh, int64_t lq, int64_t lk, int d, int block, int64_t kv_stride, bool dense,
                                 bool may_split) {
  const int64_t nk = (lk + block - 1) / block, keys = dense ? lk : std::min(nk, kv_stride) * block;
  const int64_t shares = dense ? (lk + 63) / 64 : std::min(nk, kv_stride);  // that a range can be made of
  const int most = may_split ? paged_rows_most_ranges(bh, lq, lk, block) : 1;
  CachePlan p{};
  double best = 300.0;
  for (int w = dense ? 64 : block; w <= (dense ? 128 : block); w *= 2) {
    const int64_t items = bh * ((lq + w - 1) / w), held = 256 * 4 * kAttnWavesPerSimd * 32 / w;
    auto offer = [&](int64_t r) {
      if (r < 1 || r > most || r > shares || (r > 1 && r * items > 3 * held)) return;
      if (const double t = paged_rows_time_us(bh, lq, keys, d, int(r), w); t < best) best = t, p.ranges = int(r), p.waves = w / 32;
    };
    for (const int r : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) offer(r);
    for (int i = 1; may_split && i <= 3; ++i) offer(i * held / items);
  }
  if (p.ranges == 0) {
    p = cache_attn_plan(bh, lq, lk, d, block, kv_stride, dense, may_split);
    p.ranges = std::min(p.ranges, most);
    const bool full = dense || kv_stride >= nk;
    const double rho = full ? 1.0 : double(kv_stride) / double(nk);
    auto time = [&](int ranges, int rows) {  // (with the ranges' results in fp32, not fp16)
      return attn_time_us(bh, lq, lk, d, block, rho, full, ranges, p.rotation > 0, rows) +
             (ranges > 1 ? double(bh) * double(lq) * ranges * 4 * d / 6.3e6 : 0.0);
    };
    best = 0.98 * time(p.ranges, 32 * p.waves);
    int ranges = p.ranges, rows = 32 * p.waves;
    for (int w = dense ? 64 : block; may_split && w <= (dense ? 128 : block); w *= 2) {
      const int64_t items = bh * ((lq + w - 1) / w), held = 256 * 4 * kAttnWavesPerSimd * 32 / w;
      const bool any = items <= 4 * held;
      for (int i = 1; i <= (any ? most : 3); ++i) {
        const int64_t r = any ? i : i * held / items;
        if (r < 2 || r > most || nk < r) continue;
        if (attn_grid(bh * r, (lq + w - 1) / w, 0) * 2 * w >> 32) break;  // launch limit
        if (const double t = time(int(r), w); t < best) best = t, ranges = int(r), rows = w;
      }
    }
    p.waves = rows / 32;
    p.ranges = ranges;
    if (p.rotation > 0) p.rotation = 32 * 4 * kAttnWavesPerSimd / p.waves;
  }
  const int64_t groups = (lq + 32 * p.waves - 1) / (32 * p.waves);
  p.spread_bits = attn_spread_bits(bh * p.ranges, groups, 32 * p.waves);
  p.grid = attn_grid(bh * p.ranges, groups, p.spread_bits);
  return p;
}

// The time of a call of up to 32 rows in `ranges`, us: its start and, of more than one range, its
// join; and the longer of a wave's tiles one after the other, with one work-group of four waves
// (or one of eight, or two of four) on its CU, and of all codes and scales at 6.3 TB/s.
// `uneven`: lists that may differ in length, of which the cut is by the longest.
inline double paged_token_time_us(int64_t bh, int64_t lq, int d, int64_t tiles, int ranges, int waves, bool uneven) {
  static constexpr double kTileUs[2][2][2] = {{{.82, 1.33}, {1.14, 1.83}}, {{1.2, 2.0}, {2.13, 3.17}}};
  const bool two = bh * ranges > 256;
  const double tile = kTileUs[d == 128][lq > 16][two || waves == 8];
  const double memory = double(bh) * double(tiles) * 64 * (d + d / 16) / 6.3e6 * (uneven ? 0.85 : 1.0);
  return (ranges > 1 ? 10.0 : 4.0) + (two && !uneven ? 1.5 : 0.0) + std::max(memory, tile * double(tiles) / (ranges * waves));
}

// Up to 32 rows stream the cache, in ranges of four waves each, which have a 64-key tile each at
// least, and whose work-groups fill the chip once or twice; or whole, and where whole lists leave
// a CU to one work-group it has eight waves (24 heads of 2,048 rows 12.1 us, 13.8 with four; 64 x
// 24 heads of 700 rows 47 and 33).  One token, D = 128: 24 heads of 144,512 rows 78 us with 240
// work-groups, 80 with 504; of 9,000 13.6 and 14.7; of 3,000 11.2 with 240, 15.9 whole; two
// sequences of 24 heads, 84,032 rows each 88 us with 240 and 92 with 480, 84,032 and 67,226 87
// and 84.  With 32 rows the matrix instructions want the second work-group: 24 heads of 144,512
// rows 127 us and 97, as they do at D = 64: 2 x 24 heads of 84,032 rows 61 and 51.
inline PagedPlan paged_attn_plan(int64_t bh, int64_t lq, int64_t lk, int d, int block, int64_t kv_stride, bool dense,
                                 bool may_split, bool uneven) {
  if (lq > 32) return PagedPlan{paged_rows_plan(bh, lq, lk, d, block, kv_stride, dense, may_split), 0};
  const int64_t nk = (lk + block - 1) / block, tiles = (dense ? nk : std::min(nk, kv_stride)) * (block / 64);
  PagedPlan p{{1, 1, 0, 0, 0}, tiles > 8 && bh <= 256 ? 8 : 4};
  double best = paged_token_time_us(bh, lq, d, tiles, 1, p.token_waves, uneven);
  for (int fill = 256; may_split && fill <= 512; fill += 256) {
    const int r = (int)std::min<int64_t>({fill / bh, tiles / 4, paged_token_most_ranges(bh, lk, block)});
    if (r < 2) continue;
    if (const double t = paged_token_time_us(bh, lq, d, tiles, r, 4, uneven); t < best) best = t, p.ranges = r, p.token_waves = 4;
  }
  p.grid = bh * p.ranges;
  return p;
}

// Bytes of workspace: the ranges' results in fp32, and four values per row.
inline size_t paged_part_bytes(int64_t rows, int d, int ranges) {
  return (size_t(rows * d) * ranges * 4 + 255) & ~size_t(255);
}
inline size_t paged_attn_workspace(int64_t bh, int64_t lq, int64_t lk, int d, int block) {
  const int ranges = lq > 32 ? paged_rows_most_ranges(bh, lq, lk, block) : paged_token_most_ranges(bh, lk, block);
  return ranges > 1 ? paged_part_bytes(bh * lq, d, ranges) + size_t(bh * lq) * ranges * 4 * sizeof(float) : 0;
}

// Groups of threads that share the join of a row's ranges (cache_merge_kernel; a thread loads four
// ranges at a time).  D = 128, us in one, 4 and 16 groups: 64 rows in 16 ranges 6.3, 4.0, 4.0, in 64
// 20.6, 7.5, 4.0; 2,400 in 8 4.8, 4.7, 5.2, in 16 7.2, 5.4, 6.4, in 32 12.4, 8.3, 9.9; 7,200 in 8
// 6.6, 6.8, 10.2, in 12 8.5, 8.6, 11.4.
inline int paged_join_groups(int64_t rows, int d, int ranges) {
  if (ranges <= 8 || rows * d >= 5000 * 128) return 1;
  return ranges > 16 && rows * d <= 1000 * 128 ? 16 : 4;
}

// Threads of the largest launch of a call, of which there may be fewer than 2^32.
inline int64_t paged_attn_threads(const PagedPlan& p, int64_t rows, int d) {
  if (p.waves == 1) return std::max<int64_t>(p.grid * 64 * p.token_waves, p.ranges > 1 ? rows * d * 4 : 0);
  const int64_t join = p.ranges > 1 ? rows * (d / 8) * paged_join_groups(rows, d, p.ranges) + 256 : 0;
  return std::max(p.grid * 64 * p.waves, join);
}

}  // namespace sparstar
