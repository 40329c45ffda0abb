// C ABI of the paged 4-bit key/value cache: host-side validation, workspace layout and
// launches.  As in host_api.cpp, every argument is checked before the first HIP call.
#include <math.h>

#include "paged_plan.h"
#include "rope_check.h"

using namespace sparstar;

// The pages' pool and table.
static int check_pages(const void* k, const void* v, const void* ks, const void* vs, const int32_t* pages,
                       int64_t n_table, int64_t n_pages, int B, int H, int D, int block_size) {
  if (n_table < 1 || n_table > (int64_t(1) << 30) / block_size)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "n_table must be in [1, 2^30 / block_size]");
  if (n_pages < 1 || n_pages > INT32_MAX)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "n_pages must be in [1, 2^31)");
  // (the attention counts tiles of 4,096 values in 31 bits)
  if (n_pages * block_size >= (int64_t(1) << 43) / (int64_t(H) * D))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "cache too large");
  if (!k || !v || !ks || !vs || !pages)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "the cache's four arrays and its pages must be non-null");
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | reinterpret_cast<uintptr_t>(ks) |
       reinterpret_cast<uintptr_t>(vs)) & 15u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "k_pages, v_pages, k_scale and v_scale must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(pages) & 3u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "pages must be 4-byte aligned");
  return SPARSTAR_OK;
}

static PagedArgs paged_args(const void* k_pages, const void* v_pages, const uint8_t* k_scale, const uint8_t* v_scale,
                            const int32_t* pages, int64_t n_table, int64_t n_pages, int B, int H, int64_t start,
                            int64_t L, int D, int block_size) {
  PagedArgs a{};
  a.k_pages = static_cast<uint8_t*>(const_cast<void*>(k_pages));
  a.v_pages = static_cast<uint8_t*>(const_cast<void*>(v_pages));
  a.k_scale = const_cast<uint8_t*>(k_scale);
  a.v_scale = const_cast<uint8_t*>(v_scale);
  a.pages = pages;
  a.n_table = n_table;
  a.n_pages = n_pages;
  a.l = L;
  a.start = start;
  a.b = B;
  a.heads = H;
  a.d = D;
  a.block = block_size;
  return a;
}

extern "C" int sparstar_paged_write(const void* k, sparstar_strides ks, const void* v, sparstar_strides vs, int B,
                                    int H, int64_t L, int D, int block_size, int64_t start, const int32_t* starts,
                                    const int32_t* counts, const float* table, int64_t table_rows, int pairs,
                                    int interleaved, const int32_t* positions, const int32_t* pages, int64_t n_table,
                                    int64_t n_pages, void* k_pages, void* v_pages, uint8_t* k_scale, uint8_t* v_scale,
                                    void* stream) {
  if (int rc = check_attn_sizes(B, H, L, 1, D, block_size)) return rc;
  if (int rc = check_pages(k_pages, v_pages, k_scale, v_scale, pages, n_table, n_pages, B, H, D, block_size)) return rc;
  PagedArgs a = paged_args(k_pages, v_pages, k_scale, v_scale, pages, n_table, n_pages, B, H, start, L, D, block_size);
  if (int rc = check_strides(ks, B, H, L, D, false, "k", &a.ks)) return rc;
  if (int rc = check_strides(vs, B, H, L, D, false, "v", &a.vs)) return rc;
  if (L > 0 && (!k || !v)) return report_error(SPARSTAR_ERR_INVALID_ARG, "k and v must be non-null");
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(starts) | reinterpret_cast<uintptr_t>(counts)) & 3u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "starts and counts must be 4-byte aligned");
  const int64_t cap = n_table * block_size;
  if (!starts && (start < 0 || start > cap || L > cap - start))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "the rows [start, start + L) must lie inside the pages' table");
  if (table) {
    if (int rc = check_turn(table, table_rows, pairs, interleaved, positions, D, start, L, starts != nullptr, &a.turn))
      return rc;
  } else if (positions) {
    return report_error(SPARSTAR_ERR_INVALID_ARG, "positions without a table");
  }
  if (L == 0) return clear_error();
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.starts = starts;
  a.counts = counts;
  const hipError_t e = launch_paged_write(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return report_error(SPARSTAR_ERR_HIP, hipGetErrorString(e));
  return clear_error();
}

extern "C" int sparstar_paged_read(const void* k_pages, const void* v_pages, const uint8_t* k_scale,
                                   const uint8_t* v_scale, int B, int H, int64_t start, int64_t L, int D,
                                   int block_size, const int32_t* pages, int64_t n_table, int64_t n_pages, void* k,
                                   void* v, void* stream) {
  if (int rc = check_attn_sizes(B, H, L, 1, D, block_size)) return rc;
  if (int rc = check_pages(k_pages, v_pages, k_scale, v_scale, pages, n_table, n_pages, B, H, D, block_size)) return rc;
  const int64_t cap = n_table * block_size;
  if (start < 0 || start > cap || L > cap - start)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "the rows [start, start + L) must lie inside the pages' table");
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) & 15u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "k and v must be 16-byte aligned");
  if (L == 0 || (!k && !v)) return clear_error();
  PagedArgs a = paged_args(k_pages, v_pages, k_scale, v_scale, pages, n_table, n_pages, B, H, start, L, D, block_size);
  a.k_out = static_cast<uint16_t*>(k);
  a.v_out = static_cast<uint16_t*>(v);
  const hipError_t e = launch_paged_read(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return report_error(SPARSTAR_ERR_HIP, hipGetErrorString(e));
  return clear_error();
}

extern "C" size_t sparstar_paged_attn_workspace_bytes(int B, int H, int64_t Lq, int64_t Lk, int D, int block_size) {
  if (check_attn_sizes(B, H, Lq, Lk, D, block_size) != SPARSTAR_OK) return 0;
  return paged_attn_workspace(int64_t(B) * H, Lq, Lk, D, block_size);
}

// The cut of a call of more than 32 rows with a workspace; kv_stride 0: dense.
extern "C" void sparstar_internal_paged_plan(int B, int H, int64_t Lq, int64_t Lk, int D, int block_size,
                                             int64_t kv_stride, int64_t* out) {
  const CachePlan p = paged_rows_plan(int64_t(B) * H, Lq, Lk, D, block_size, kv_stride, kv_stride == 0, true);
  out[0] = p.waves, out[1] = p.ranges, out[2] = p.rotation;
}

extern "C" int sparstar_internal_paged_ranges(int B, int H, int64_t Lq, int64_t Lk, int D, int block_size,
                                              int64_t kv_stride) {
  if (check_attn_sizes(B, H, Lq, Lk, D, block_size) != SPARSTAR_OK) return 1;
  const bool dense = kv_stride == 0;
  int most = 1;  // of lists of even and of uneven lengths
  for (const bool uneven : {false, true})
    most = std::max(most, paged_attn_plan(int64_t(B) * H, Lq, Lk, D, block_size, kv_stride, dense, true, uneven).ranges);
  return most;
}

static int paged_attn_common(const void* q, const void* k_pages, const void* v_pages, const uint8_t* k_scale,
                             const uint8_t* v_scale, int B, int H, int64_t Lq, int64_t Lk, int D, int block_size,
                             const int32_t* pages, int64_t n_table, int64_t n_pages, const int32_t* lens,
                             const int32_t* kv_num_blocks, const int32_t* kv_indices, int kv_stride,
                             float softmax_scale, void* o, float* lse, void* workspace, size_t workspace_bytes,
                             void* stream, bool dense) {
  if (int rc = check_attn_sizes(B, H, Lq, Lk, D, block_size)) return rc;
  if (int rc = check_pages(k_pages, v_pages, k_scale, v_scale, pages, n_table, n_pages, B, H, D, block_size)) return rc;
  if (Lk > n_table * block_size)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "Lk exceeds the rows of the pages' table");
  if (Lq > 0 && (!q || !o)) return report_error(SPARSTAR_ERR_INVALID_ARG, "q and o must be non-null");
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(o)) & 15u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "q and o must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(lens)) & 3u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "lse and lens must be 4-byte aligned");
  if (!dense && Lq > 0) {
    if (!kv_num_blocks || !kv_indices)
      return report_error(SPARSTAR_ERR_INVALID_ARG, "kv_num_blocks and kv_indices must be non-null");
    if (kv_stride < 1 || kv_stride > (1 << 28))
      return report_error(SPARSTAR_ERR_INVALID_ARG, "kv_stride must be in [1, 2^28]");
  }
  if (!(softmax_scale == softmax_scale) || isinf(softmax_scale))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "softmax_scale must be finite");
  const int64_t bh = int64_t(B) * H;
  const PagedPlan plan =
      paged_attn_plan(bh, Lq, Lk, D, block_size, dense ? 0 : kv_stride, dense, workspace != nullptr,
                      !dense || (lens != nullptr && B > 1));
  if (paged_attn_threads(plan, bh * Lq, D) >= int64_t(1) << 32)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "too many query rows and heads for one call");
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
    return report_error(SPARSTAR_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (workspace && workspace_bytes < paged_attn_workspace(bh, Lq, Lk, D, block_size))
    return report_error(SPARSTAR_ERR_WORKSPACE, "workspace is smaller than sparstar_paged_attn_workspace_bytes");
  if (Lq == 0) return clear_error();
  const double sc = softmax_scale > 0.f ? double(softmax_scale) : 1.0 / sqrt(double(D));
  PagedAttnArgs a{};
  a.q = static_cast<const uint16_t*>(q);
  a.k_cache = static_cast<const uint8_t*>(k_pages);
  a.v_cache = static_cast<const uint8_t*>(v_pages);
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.pages = pages;
  a.n_table = n_table;
  a.n_pages = n_pages;
  a.lens = lens;
  a.kv_num_blocks = kv_num_blocks;
  a.kv_indices = kv_indices;
  a.o = static_cast<uint16_t*>(o);
  a.lse = lse;
  a.lq = Lq;
  a.lk = Lk;
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
  a.waves = plan.waves;
  a.token_waves = plan.token_waves;
  a.join_groups = paged_join_groups(bh * Lq, D, plan.ranges);
  if (plan.ranges > 1) {
    a.part32 = static_cast<float*>(workspace);
    a.part_o = static_cast<uint16_t*>(workspace);
    a.part_meta = reinterpret_cast<float*>(static_cast<char*>(workspace) + paged_part_bytes(bh * Lq, D, plan.ranges));
  }
  const hipError_t e = launch_paged_attn(a, D, dense, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return report_error(SPARSTAR_ERR_HIP, hipGetErrorString(e));
  return clear_error();
}

extern "C" int sparstar_paged_sparse_attn_fwd(const void* q, const void* k_pages, const void* v_pages,
                                              const uint8_t* k_scale, const uint8_t* v_scale, int B, int H, int64_t Lq,
                                              int64_t Lk, int D, int block_size, const int32_t* pages, int64_t n_table,
                                              int64_t n_pages, const int32_t* lens, const int32_t* kv_num_blocks,
                                              const int32_t* kv_indices, int kv_stride, float softmax_scale, void* o,
                                              float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  return paged_attn_common(q, k_pages, v_pages, k_scale, v_scale, B, H, Lq, Lk, D, block_size, pages, n_table, n_pages,
                           lens, kv_num_blocks, kv_indices, kv_stride, softmax_scale, o, lse, workspace,
                           workspace_bytes, stream, false);
}

extern "C" int sparstar_paged_dense_attn_fwd(const void* q, const void* k_pages, const void* v_pages,
                                             const uint8_t* k_scale, const uint8_t* v_scale, int B, int H, int64_t Lq,
                                             int64_t Lk, int D, int block_size, const int32_t* pages, int64_t n_table,
                                             int64_t n_pages, const int32_t* lens, float softmax_scale, void* o,
                                             float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  return paged_attn_common(q, k_pages, v_pages, k_scale, v_scale, B, H, Lq, Lk, D, block_size, pages, n_table, n_pages,
                           lens, nullptr, nullptr, 0, softmax_scale, o, lse, workspace, workspace_bytes, stream, true);
}
