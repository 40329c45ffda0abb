// C ABI of the attention's gradients: host-side validation, workspace layout and
// launches.  As in host_api.cpp, every argument is checked before the first HIP call.
#include <math.h>

#include "../../include/sparstar.h"
#include "bwd_plan.h"
#include "host_internal.h"

using namespace sparstar;

extern "C" size_t sparstar_attn_bwd_workspace_bytes(int B, int H, int64_t Lq, int64_t Lk, int D, int block_size) {
  if (check_attn_sizes(B, H, Lq, Lk, D, block_size) != SPARSTAR_OK) return 0;
  const int64_t bh = int64_t(B) * H;
  return std::max(attn_bwd_plan(bh, Lq, Lk, D, block_size, false).total,
                  attn_bwd_plan(bh, Lq, Lk, D, block_size, true).total);
}

extern "C" void sparstar_internal_bwd_plan(int B, int H, int64_t Lq, int64_t Lk, int D, int block_size, int dense,
                                           int64_t* out) {
  const BwdPlan p = attn_bwd_plan(int64_t(B) * H, Lq, Lk, D, block_size, dense != 0);
  out[0] = p.dq_ranges;
  out[1] = p.dkv_ranges;
  if (p.slots > 0) {  // pieces of a key block that every query lists, if all lists are full
    const int64_t nq = (Lq + block_size - 1) / block_size, nk = (Lk + block_size - 1) / block_size;
    const int64_t most = attn_bwd_piece_max(int64_t(B) * H, nq, nk, block_size);
    out[1] = (nq + most - 1) / most;
  }
}

extern "C" void sparstar_internal_bwd_pieces(int B, int H, int64_t Lq, int64_t Lk, int D, int block_size,
                                             int64_t kv_stride, int64_t* out) {
  const int64_t bh = int64_t(B) * H, nq = (Lq + block_size - 1) / block_size, nk = (Lk + block_size - 1) / block_size;
  const BwdPlan p = attn_bwd_plan(bh, Lq, Lk, D, block_size, false);
  const BwdPieces c = attn_bwd_pieces(p, bh, nq, nk, std::min(kv_stride, nk), block_size);
  out[0] = c.list_min;
  out[1] = c.piece_max;
  out[2] = int64_t(p.count);
  out[3] = int64_t(p.pieces);
}

static int bwd_common(const void* q, const void* k, const void* v, const void* o, const float* lse, const void* d_o,
                      const float* d_lse, int B, int H, int64_t Lq, int64_t Lk, int D, int block_size,
                      const int32_t* kv_num_blocks, const int32_t* kv_indices, int kv_stride, float softmax_scale,
                      void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes, void* stream,
                      bool dense) {
  if (int rc = check_attn_sizes(B, H, Lq, Lk, D, block_size)) return rc;
  if (!k || !v || !dk || !dv || (Lq > 0 && (!q || !o || !lse || !d_o || !dq)))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "q, k, v, o, lse, d_o, dq, dk and dv must be non-null");
  uintptr_t mis = 0;
  for (const void* p : {q, k, v, o, d_o, (const void*)dq, (const void*)dk, (const void*)dv})
    mis |= reinterpret_cast<uintptr_t>(p);
  if (mis & 15u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "q, k, v, o, d_o, dq, dk and dv must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(d_lse)) & 3u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "lse and d_lse must be 4-byte aligned");
  if (!dense && Lq > 0) {
    if (!kv_num_blocks || !kv_indices)
      return report_error(SPARSTAR_ERR_INVALID_ARG, "kv_num_blocks and kv_indices must be non-null");
    if (kv_stride < 1) return report_error(SPARSTAR_ERR_INVALID_ARG, "kv_stride must be >= 1");
  }
  if (!(softmax_scale == softmax_scale) || isinf(softmax_scale))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "softmax_scale must be finite");
  // (lse / s has to stay finite)
  if (softmax_scale > 0.f && softmax_scale < 1e-30f)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "softmax_scale must be at least 1e-30, or <= 0 for D^-1/2");
  const int64_t bh = int64_t(B) * H;
  const BwdPlan plan = attn_bwd_plan(bh, Lq, Lk, D, block_size, dense);
  if (!workspace && plan.total > 0) return report_error(SPARSTAR_ERR_WORKSPACE, "workspace is null");
  if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0)
    return report_error(SPARSTAR_ERR_WORKSPACE, "workspace must be 256-byte aligned");
  if (workspace_bytes < plan.total)
    return report_error(SPARSTAR_ERR_WORKSPACE, "workspace is smaller than sparstar_attn_bwd_workspace_bytes");
  const double sc = softmax_scale > 0.f ? double(softmax_scale) : 1.0 / sqrt(double(D));
  BwdArgs a{};
  a.q = static_cast<const uint16_t*>(q);
  a.o = static_cast<const uint16_t*>(o);
  a.d_o = static_cast<const uint16_t*>(d_o);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.lse = lse;
  a.dlse = d_lse;
  a.dq = static_cast<uint16_t*>(dq);
  a.dk = static_cast<uint16_t*>(dk);
  a.dv = static_cast<uint16_t*>(dv);
  a.kv_num_blocks = kv_num_blocks;
  a.kv_indices = kv_indices;
  a.lq = Lq;
  a.lk = Lk;
  a.bh = int(bh);
  a.n_q = int((Lq + block_size - 1) / block_size);
  a.n_k = int((Lk + block_size - 1) / block_size);
  a.stride = kv_stride;
  a.block = block_size;
  a.scale = float(sc);
  a.inv_scale = float(1.0 / sc);
  a.scale_log2 = float(sc * 1.4426950408889634074);
  a.n_words = (a.n_q + 31) / 32;
  char* ws = static_cast<char*>(workspace);
  a.stats = reinterpret_cast<float*>(ws + plan.stats);
  a.bits = reinterpret_cast<uint32_t*>(ws + plan.bits);
  a.part = reinterpret_cast<float*>(ws + plan.part);
  a.part_kv = reinterpret_cast<float*>(ws + plan.part_kv);
  a.dq_ranges = plan.dq_ranges;
  a.dkv_ranges = plan.dkv_ranges;
  if (!dense && (plan.rounds || plan.slots > 0)) {
    const BwdPieces c = attn_bwd_pieces(plan, bh, a.n_q, a.n_k, std::min(kv_stride, a.n_k), block_size);
    a.list_min = c.list_min;
    a.piece_max = c.piece_max;
    a.most_pieces = c.most_pieces;
    a.piece_count = reinterpret_cast<int32_t*>(ws + plan.count);
    a.pieces = reinterpret_cast<BwdPiece*>(ws + plan.pieces);
    a.listed = reinterpret_cast<uint8_t*>(ws + plan.listed);
    a.part_piece = reinterpret_cast<float*>(ws + plan.part_piece);
  }
  if (attn_bwd_threads(plan, bh, Lq, Lk, D, block_size, dense, a.most_pieces) >= int64_t(1) << 32)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "too many rows and heads for one call");
  const hipError_t e = launch_attn_bwd(a, D, dense, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return report_error(SPARSTAR_ERR_HIP, hipGetErrorString(e));
  return clear_error();
}

extern "C" int sparstar_sparse_attn_bwd(const void* q, const void* k, const void* v, const void* o, const float* lse,
                                        const void* d_o, const float* d_lse, int B, int H, int64_t Lq, int64_t Lk,
                                        int D, int block_size, const int32_t* kv_num_blocks, const int32_t* kv_indices,
                                        int kv_stride, float softmax_scale, void* dq, void* dk, void* dv,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  return bwd_common(q, k, v, o, lse, d_o, d_lse, B, H, Lq, Lk, D, block_size, kv_num_blocks, kv_indices, kv_stride,
                    softmax_scale, dq, dk, dv, workspace, workspace_bytes, stream, false);
}

extern "C" int sparstar_dense_attn_bwd(const void* q, const void* k, const void* v, const void* o, const float* lse,
                                       const void* d_o, const float* d_lse, int B, int H, int64_t Lq, int64_t Lk,
                                       int D, int block_size, float softmax_scale, void* dq, void* dk, void* dv,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  return bwd_common(q, k, v, o, lse, d_o, d_lse, B, H, Lq, Lk, D, block_size, nullptr, nullptr, 0, softmax_scale, dq,
                    dk, dv, workspace, workspace_bytes, stream, true);
}
