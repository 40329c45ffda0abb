// How a gradient call is cut up (host code): the key ranges of the dQ pass, the
// query ranges of the dK/dV pass, and the workspace that follows from them.  The
// kernels (attn_bwd.hip) take the cut through BwdArgs.
#pragma once

#include <algorithm>

#include "launch.h"

namespace sparstar {

struct BwdPlan {
  int dq_ranges, dkv_ranges;
  bool rounds;  // the dK/dV pass has more work-groups than the chip holds
  size_t stats, bits, part, total;  // byte offsets of the workspace's regions, and its size
};

constexpr int kBwdMaxRanges = 16;

// Ranges of one pass: work-groups of `rows` rows that each walk `tiles` tiles, of
// which the chip holds `held` at once.  Few work-groups leave CUs idle, so the walk
// is cut until they fill the chip, as long as a range keeps 16 tiles.
inline int bwd_ranges(int64_t groups, int64_t held, int64_t tiles) {
  int r = 1;
  while (r < kBwdMaxRanges && groups * r < 2 * held && tiles >= 32 * r) r *= 2;
  return r;
}

inline BwdPlan attn_bwd_plan(int64_t bh, int64_t lq, int64_t lk, int d, int block, bool dense) {
  const int rows = dense ? 128 : block, waves = rows / 32, tile = attn_tile_keys(d);
  const int64_t nq = (lq + block - 1) / block, nk = (lk + block - 1) / block;
  BwdPlan p{};
  p.dq_ranges = bwd_ranges(bh * ((lq + rows - 1) / rows), 256 * 8 / waves, (lk + tile - 1) / tile);
  const int64_t key_groups = bh * ((lk + rows - 1) / rows), held = 256 * (d == 128 ? 4 : 8) / waves;
  p.dkv_ranges = bwd_ranges(key_groups, held, (lq + tile - 1) / tile);
  // (the sparse walk is cut at whole words of 32 query blocks)
  if (!dense) p.dkv_ranges = (int)std::min<int64_t>(p.dkv_ranges, std::max<int64_t>(1, (nq + 31) / 32));
  p.rounds = key_groups * p.dkv_ranges > held;
  auto align = [](size_t x) { return (x + 255) & ~size_t(255); };
  p.stats = 0;
  p.bits = align(size_t(bh * nq * block) * 2 * sizeof(float));
  p.part = p.bits + (dense ? 0 : align(size_t(bh * nk * ((nq + 31) / 32)) * sizeof(uint32_t)));
  const size_t dq = p.dq_ranges > 1 ? size_t(bh * lq * d) * p.dq_ranges * sizeof(float) : 0;
  const size_t dkv = p.dkv_ranges > 1 ? 2 * size_t(bh * lk * d) * p.dkv_ranges * sizeof(float) : 0;
  p.total = p.part + std::max(dq, dkv);
  return p;
}

}  // namespace sparstar
