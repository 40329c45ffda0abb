// How an attention call over the paged cache is cut up (host code).
#pragma once

#include "cache_plan.h"

namespace sparstar {

struct PagedPlan {
  int waves;   // 1: the kernels for up to 32 rows
  int ranges;  // of each list's entries
  int rotation, spread_bits;
  int64_t grid;
};

inline PagedPlan paged_attn_plan(int64_t bh, int64_t lq, int64_t lk, int d, int block, int64_t kv_stride, bool dense,
                                 bool may_split) {
  return PagedPlan{1, 1, 0, 0, bh * lq};
}

// Bytes of workspace for the most ranges that these sizes are cut into.
inline size_t paged_attn_workspace(int64_t bh, int64_t lq, int64_t lk, int d, int block) { return 0; }

// Threads of the largest launch of a call, of which there may be fewer than 2^32.
inline int64_t paged_attn_threads(const PagedPlan& p, int64_t rows, int d) { return p.grid * 64; }

}  // namespace sparstar
