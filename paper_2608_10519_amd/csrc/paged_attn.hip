// Attention over the paged 4-bit key/value cache (paged.hip), dense or over block lists.
#include "cache_attn_kernel.h"

namespace sparstar {

// One wave per query row: 64 keys at a time, a key per lane for the scores, a pair of
// channels per lane (D = 64: a channel) for the sum.
template <int D, bool DENSE>
__global__ __launch_bounds__(64) void paged_row_kernel(PagedAttnArgs a) {
  __shared__ float qs[D];
  constexpr int CPL = D / 64;  // channels per lane
  const int lane = threadIdx.x;
  const int64_t at = blockIdx.x, bh = at / a.lq, row = at - bh * a.lq, b = bh / a.heads, h = bh - b * a.heads;
  for (int d = lane; d < D; d += 64) qs[d] = bf16_lo(a.q[at * D + d]);
  __syncthreads();
  int64_t len = a.lk;
  if (a.lens != nullptr) {
    const int n = a.lens[b];
    len = n < 0 ? 0 : (n < a.lk ? n : a.lk);
  }
  const int n_blk = (int)((len + a.block - 1) / a.block);
  int n = n_blk;
  const int32_t* list = nullptr;
  if constexpr (!DENSE) {
    const int64_t r = bh * a.n_q + row / a.block;
    n = a.kv_num_blocks[r];
    n = n < 0 ? 0 : (n > a.stride ? a.stride : n);
    list = a.kv_indices + r * a.stride;
  }
  float m = -INFINITY, l = 0.f, le = 0.f, o[CPL] = {};
  for (int e = 0; e < n; ++e) {
    const int j = DENSE ? e : list[e];
    if (j < 0 || j >= n_blk) continue;
    const int64_t page = a.pages[b * a.n_table + j];
    if (page < 0 || page >= a.n_pages) continue;
    for (int sub = 0; sub < a.block; sub += 64) {
      const int64_t left = len - ((int64_t)j * a.block + sub);
      if (left <= 0) break;
      const int64_t r0 = (page * a.heads + h) * a.block + sub;
      float s = -INFINITY;
      if (lane < left) {
        s = 0.f;
        const uint32_t* w = reinterpret_cast<const uint32_t*>(a.k_cache + (r0 + lane) * (D / 2));
        for (int c = 0; c < D / 8; ++c) {
          const float sc = __uint_as_float((uint32_t)a.k_scale[(r0 + lane) * (D / 32) + c / 4] << 23);
          const auto u0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[c], sc, 0);
          const auto u1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[c], sc, 1);
          const auto u2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[c], sc, 2);
          const auto u3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[c], sc, 3);
          const float* q = qs + 8 * c;
          s += u0[0] * q[0] + u0[1] * q[1] + u1[0] * q[2] + u1[1] * q[3];
          s += u2[0] * q[4] + u2[1] * q[5] + u3[0] * q[6] + u3[1] * q[7];
        }
        s *= a.scale_log2;
      }
      float mx = s;
      for (int i = 32; i > 0; i /= 2) mx = fmaxf(mx, __shfl_xor(mx, i));
      const float mn = fmaxf(m, mx), alpha = mn == -INFINITY ? 0.f : exp2f(m - mn);
      const float p = mn == -INFINITY ? 0.f : exp2f(s - mn);
      m = mn;
      l = l * alpha + p;
      for (int i = 0; i < CPL; ++i) o[i] *= alpha;
      const int keys = left < 64 ? (int)left : 64;
      for (int k = 0; k < keys; ++k) {
        const float pk = __shfl(p, k);
        const uint8_t* w = a.v_cache + (r0 + k) * (D / 2);
        for (int i = 0; i < CPL; ++i) {
          const int d = CPL * lane + i;
          const float sc = __uint_as_float((uint32_t)a.v_scale[(r0 + k) * (D / 32) + d / 32] << 23);
          const auto u = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)w[d / 2], sc, 0);
          o[i] = fmaf(pk, d % 2 ? u[1] : u[0], o[i]);
        }
      }
    }
  }
  for (int i = 32; i > 0; i /= 2) l += __shfl_xor(l, i);
  const float inv = l == 0.f ? 0.f : 1.f / l;
  for (int i = 0; i < CPL; ++i)
    a.o[at * D + CPL * lane + i] = (uint16_t)pack2_bf16(o[i] * inv, 0.f);
  if (a.lse != nullptr && lane == 0) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994530942f;
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, int d, int waves, bool dense, hipStream_t stream) {
  const int64_t rows = (int64_t)a.bh * a.lq;
  if (waves > 1) {
    if (d == 128) return dense ? launch_rows<128, true, Codes4>(a, waves, stream) : launch_rows<128, false, Codes4>(a, waves, stream);
    return dense ? launch_rows<64, true, Codes4>(a, waves, stream) : launch_rows<64, false, Codes4>(a, waves, stream);
  }
  if (d == 128 && dense) paged_row_kernel<128, true><<<rows, 64, 0, stream>>>(a);
  else if (d == 128) paged_row_kernel<128, false><<<rows, 64, 0, stream>>>(a);
  else if (dense) paged_row_kernel<64, true><<<rows, 64, 0, stream>>>(a);
  else paged_row_kernel<64, false><<<rows, 64, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace sparstar
