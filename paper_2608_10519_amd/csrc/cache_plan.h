// How an attention call over the 8-bit cache is cut up (host code): waves per
// work-group, and ranges of each list.  The kernel (cache_attn.hip) takes the cut
// through CacheAttnArgs.
#pragma once

#include <algorithm>

#include "launch.h"

namespace sparstar {

struct CachePlan {
  int waves;   // of a work-group, 32 query rows each
  int ranges;  // of each list's entries
};

constexpr int kCacheMaxRanges = 16, kCacheMaxTokenRanges = 64;

// `entries`: key blocks that a list can name.
inline CachePlan cache_attn_plan(int64_t bh, int64_t lq, int64_t entries, int block, bool dense) {
  CachePlan p{dense ? (lq <= 64 ? 2 : 4) : block / 32, 1};
  if (lq <= 32) {
    // A few rows stream the cache: single waves, each with its own ring of tiles (32 KB,
    // five to a CU), as many as the chip holds while each has two blocks to read.
    p.waves = 1;
    const int64_t want = (256 * 5 + bh - 1) / bh;
    p.ranges = (int)std::max<int64_t>(1, std::min<int64_t>({want, entries / 2, kCacheMaxTokenRanges}));
    return p;
  }
  const int64_t groups = bh * ((lq + 32 * p.waves - 1) / (32 * p.waves)), held = 256 * 8 / p.waves;
  while (p.ranges < kCacheMaxRanges && groups * p.ranges < 2 * held && entries >= 16 * p.ranges) p.ranges *= 2;
  return p;
}

inline size_t cache_part_o_bytes(int64_t rows, int d, int ranges) {
  return (size_t(rows * d) * ranges * sizeof(float) + 255) & ~size_t(255);
}

inline size_t cache_attn_workspace(int64_t rows, int d, int ranges) {
  return ranges > 1 ? cache_part_o_bytes(rows, d, ranges) + size_t(rows) * ranges * 4 * sizeof(float) : 0;
}

}  // namespace sparstar
