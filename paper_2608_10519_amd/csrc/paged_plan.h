// How an attention call over the paged cache is cut up (host code).
#pragma once

#include "cache_plan.h"

namespace sparstar {

// As for the 8-bit cache (waves == 1: the kernels for up to 32 rows).
using PagedPlan = CachePlan;

inline PagedPlan paged_attn_plan(int64_t bh, int64_t lq, int64_t lk, int d, int block, int64_t kv_stride, bool dense,
                                 bool may_split) {
  if (lq > 32) return cache_attn_plan(bh, lq, lk, d, block, kv_stride, dense, may_split);
  return PagedPlan{1, 1, 0, 0, bh * lq};
}

// Bytes of workspace for the most ranges that these sizes are cut into.
inline size_t paged_attn_workspace(int64_t bh, int64_t lq, int64_t lk, int d, int block) {
  if (lq > 32) return cache_attn_workspace(bh * lq, d, cache_attn_most_ranges(bh, lq, lk, block));
  return 0;
}

// Threads of the largest launch of a call, of which there may be fewer than 2^32.
inline int64_t paged_attn_threads(const PagedPlan& p, int64_t rows, int d) {
  if (p.waves == 1) return p.grid * 64;
  return cache_attn_threads(p, rows, d);
}

}  // namespace sparstar
