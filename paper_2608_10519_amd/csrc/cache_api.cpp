// C ABI of the 8-bit key/value cache: host-side validation, workspace layout and
// launches.  As in host_api.cpp, every argument is checked before the first HIP call.
#include <math.h>

#include "../../include/sparstar.h"
#include "cache_plan.h"
#include "host_internal.h"

using namespace sparstar;

// A cache's capacity and pointers.
static int check_cache(const void* k, const void* v, const void* ks, const void* vs, int64_t cap, int64_t bh, int D) {
  if (cap < 1 || cap > (int64_t(1) << 30))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "the cache's capacity must be in [1, 2^30]");
  if (bh * cap * D > (int64_t(1) << 46)) return report_error(SPARSTAR_ERR_INVALID_ARG, "cache too large");
  if (!k || !v || !ks || !vs)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "the cache's four arrays must be non-null");
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "k_cache and v_cache must be 16-byte aligned");
  return SPARSTAR_OK;
}

extern "C" int sparstar_cache_write(const void* k, const void* v, int B, int H, int64_t L, int D, int block_size,
                                    int64_t start, const int32_t* starts, const int32_t* counts, int64_t cap,
                                    void* k_cache, void* v_cache, uint8_t* k_scale, uint8_t* v_scale, void* stream) {
  if (int rc = check_attn_sizes(B, H, L, 1, D, block_size)) return rc;
  const int64_t bh = int64_t(B) * H;
  if (int rc = check_cache(k_cache, v_cache, k_scale, v_scale, cap, bh, D)) return rc;
  if (L > 0 && (!k || !v)) return report_error(SPARSTAR_ERR_INVALID_ARG, "k and v must be non-null");
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(starts) | reinterpret_cast<uintptr_t>(counts)) & 3u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "starts and counts must be 4-byte aligned");
  if (!starts && (start < 0 || start > cap || L > cap - start))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "the rows [start, start + L) must lie inside [0, cap)");
  if (L == 0) return clear_error();
  CacheWriteArgs a{};
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.k_cache = static_cast<uint8_t*>(k_cache);
  a.v_cache = static_cast<uint8_t*>(v_cache);
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.starts = starts;
  a.counts = counts;
  a.l = L;
  a.cap = cap;
  a.start = start;
  a.bh = int(bh);
  a.heads = H;
  // (with the first row known, only the blocks that the rows do touch)
  a.n_blocks = int(starts ? (L + block_size - 2) / block_size + 1
                          : (start + L - 1) / block_size - start / block_size + 1);
  const hipError_t e = launch_cache_write(a, D, block_size, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return report_error(SPARSTAR_ERR_HIP, hipGetErrorString(e));
  return clear_error();
}

extern "C" int sparstar_cache_read(const void* k_cache, const void* v_cache, const uint8_t* k_scale,
                                   const uint8_t* v_scale, int B, int H, int64_t start, int64_t L, int64_t cap, int D,
                                   int block_size, void* k, void* v, void* stream) {
  if (int rc = check_attn_sizes(B, H, L, 1, D, block_size)) return rc;
  const int64_t bh = int64_t(B) * H;
  if (int rc = check_cache(k_cache, v_cache, k_scale, v_scale, cap, bh, D)) return rc;
  if (start < 0 || start > cap || L > cap - start)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "the rows [start, start + L) must lie inside [0, cap)");
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
  if (L == 0 || (!k && !v)) return clear_error();
  CacheReadArgs a{};
  a.k_cache = static_cast<const uint8_t*>(k_cache);
  a.v_cache = static_cast<const uint8_t*>(v_cache);
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.k_out = static_cast<uint16_t*>(k);
  a.v_out = static_cast<uint16_t*>(v);
  a.l = L;
  a.cap = cap;
  a.start = start;
  a.bh = int(bh);
  a.d = D;
  a.block = block_size;
  const hipError_t e = launch_cache_read(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return report_error(SPARSTAR_ERR_HIP, hipGetErrorString(e));
  return clear_error();
}

extern "C" size_t sparstar_cache_attn_workspace_bytes(int B, int H, int64_t Lq, int64_t Lk, int D, int block_size) {
  if (check_attn_sizes(B, H, Lq, Lk, D, block_size) != SPARSTAR_OK) return 0;
  return cache_attn_workspace(int64_t(B) * H * Lq, D, cache_attn_most_ranges(int64_t(B) * H, Lq, Lk, block_size));
}

extern "C" void sparstar_internal_cache_plan(int B, int H, int64_t Lq, int64_t Lk, int D, int block_size,
                                             int64_t kv_stride, int64_t* out) {
  const CachePlan p = cache_attn_plan(int64_t(B) * H, Lq, Lk, D, block_size, kv_stride, kv_stride == 0, true);
  out[0] = p.waves;
  // parts of a list that are joined: ranges, and the waves' shares of them
  const int64_t nk = (Lk + block_size - 1) / block_size, entries = kv_stride == 0 ? nk : std::min(nk, kv_stride);
  out[1] = p.waves == 1 ? std::min<int64_t>(entries, int64_t(p.ranges) * kTokenWaves) : p.ranges;
}

// Ranges of such a call with a workspace; kv_stride 0: dense.  1: it would not use one.
extern "C" int sparstar_internal_cache_ranges(int B, int H, int64_t Lq, int64_t Lk, int D, int block_size,
                                              int64_t kv_stride) {
  if (check_attn_sizes(B, H, Lq, Lk, D, block_size) != SPARSTAR_OK) return 1;
  return cache_attn_plan(int64_t(B) * H, Lq, Lk, D, block_size, kv_stride, kv_stride == 0, true).ranges;
}

static int cache_attn_common(const void* q, const void* k_cache, const void* v_cache, const uint8_t* k_scale,
                             const uint8_t* v_scale, int B, int H, int64_t Lq, int64_t Lk, int64_t cap, int D,
                             int block_size, const int32_t* lens, const int32_t* kv_num_blocks,
                             const int32_t* kv_indices, int kv_stride, float softmax_scale, void* o, float* lse,
                             void* workspace, size_t workspace_bytes, void* stream, bool dense) {
  if (int rc = check_attn_sizes(B, H, Lq, Lk, D, block_size)) return rc;
  const int64_t bh = int64_t(B) * H;
  if (int rc = check_cache(k_cache, v_cache, k_scale, v_scale, cap, bh, D)) return rc;
  if (Lk > cap) return report_error(SPARSTAR_ERR_INVALID_ARG, "Lk exceeds the cache's capacity");
  if (Lq > 0 && (!q || !o)) return report_error(SPARSTAR_ERR_INVALID_ARG, "q and o must be non-null");
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(o)) & 15u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "q and o must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(lens)) & 3u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "lse and lens must be 4-byte aligned");
  if (!dense && Lq > 0) {
    if (!kv_num_blocks || !kv_indices)
      return report_error(SPARSTAR_ERR_INVALID_ARG, "kv_num_blocks and kv_indices must be non-null");
    if (kv_stride < 1) return report_error(SPARSTAR_ERR_INVALID_ARG, "kv_stride must be >= 1");
  }
  if (!(softmax_scale == softmax_scale) || isinf(softmax_scale))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "softmax_scale must be finite");
  const CachePlan plan =
      cache_attn_plan(bh, Lq, Lk, D, block_size, dense ? 0 : kv_stride, dense, workspace != nullptr);
  if (cache_attn_threads(plan, bh * Lq, D) >= int64_t(1) << 32)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "too many query rows and heads for one call");
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
    return report_error(SPARSTAR_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (workspace &&
      workspace_bytes < cache_attn_workspace(bh * Lq, D, cache_attn_most_ranges(bh, Lq, Lk, block_size)))
    return report_error(SPARSTAR_ERR_WORKSPACE, "workspace is smaller than sparstar_cache_attn_workspace_bytes");
  if (Lq == 0) return clear_error();
  const double sc = softmax_scale > 0.f ? double(softmax_scale) : 1.0 / sqrt(double(D));
  CacheAttnArgs a{};
  a.q = static_cast<const uint16_t*>(q);
  a.k_cache = static_cast<const uint8_t*>(k_cache);
  a.v_cache = static_cast<const uint8_t*>(v_cache);
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.lens = lens;
  a.kv_num_blocks = kv_num_blocks;
  a.kv_indices = kv_indices;
  a.o = static_cast<uint16_t*>(o);
  a.lse = lse;
  a.lq = Lq;
  a.lk = Lk;
  a.cap = cap;
  a.bh = int(bh);
  a.heads = H;
  a.block = block_size;
  a.n_q = int((Lq + block_size - 1) / block_size);
  a.stride = kv_stride;
  a.scale_log2 = float(sc * 1.4426950408889634074);
  a.ranges = plan.ranges;
  a.rotation = plan.rotation;
  a.spread_bits = plan.spread_bits;
  a.grid = plan.grid;
  if (plan.ranges > 1) {
    a.part_o = static_cast<uint16_t*>(workspace);
    a.part_meta = reinterpret_cast<float*>(static_cast<char*>(workspace) + cache_part_o_bytes(bh * Lq, D, plan.ranges));
  }
  const hipError_t e = launch_cache_attn(a, D, plan.waves, dense, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return report_error(SPARSTAR_ERR_HIP, hipGetErrorString(e));
  return clear_error();
}

extern "C" int sparstar_cache_sparse_attn_fwd(const void* q, const void* k_cache, const void* v_cache,
                                              const uint8_t* k_scale, const uint8_t* v_scale, int B, int H, int64_t Lq,
                                              int64_t Lk, int64_t cap, int D, int block_size, const int32_t* lens,
                                              const int32_t* kv_num_blocks, const int32_t* kv_indices, int kv_stride,
                                              float softmax_scale, void* o, float* lse, void* workspace,
                                              size_t workspace_bytes, void* stream) {
  return cache_attn_common(q, k_cache, v_cache, k_scale, v_scale, B, H, Lq, Lk, cap, D, block_size, lens,
                           kv_num_blocks, kv_indices, kv_stride, softmax_scale, o, lse, workspace, workspace_bytes,
                           stream, false);
}

extern "C" int sparstar_cache_dense_attn_fwd(const void* q, const void* k_cache, const void* v_cache,
                                             const uint8_t* k_scale, const uint8_t* v_scale, int B, int H, int64_t Lq,
                                             int64_t Lk, int64_t cap, int D, int block_size, const int32_t* lens,
                                             float softmax_scale, void* o, float* lse, void* workspace,
                                             size_t workspace_bytes, void* stream) {
  return cache_attn_common(q, k_cache, v_cache, k_scale, v_scale, B, H, Lq, Lk, cap, D, block_size, lens, nullptr,
                           nullptr, 0, softmax_scale, o, lse, workspace, workspace_bytes, stream, true);
}
