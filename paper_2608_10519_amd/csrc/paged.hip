// The paged 4-bit key/value cache: quantising writes, with the rotation of the keys on the
// way, and exact reads.
//
// A value is code * 2^e: an e2m1 code, and one exponent for 32 channels of a token.  A power
// of two rounds nothing, so a code is the value's nearest e2m1 number and code * 2^e is exact
// in bf16.  e is the least integer with amax 2^-e <= 6, the largest e2m1 number: nothing
// finite saturates (but past 6 * 2^125).  Tokens have scales of their own, so a write touches
// no row but its own, whatever its page holds.
#include "rope_device.h"

namespace sparstar {

// One thread per (K or V, token, chunk of 8 channels, group of heads); four neighbouring
// threads share a scale.
template <bool INTERLEAVED>
__global__ __launch_bounds__(256) void paged_write_kernel(PagedArgs a, int groups, int per_group) {
  const int cpr = a.d / 8;
  const int64_t i = group_of_rows() * 256 + threadIdx.x;
  const int64_t tokens = (int64_t)a.b * a.l, w = i / cpr;
  if (w >= 2 * tokens * groups) return;  // (whole rows of cpr threads: whole groups of four)
  const int c = (int)(i - w * cpr);
  const int g2 = (int)(w / tokens), is_v = g2 >= groups, g = is_v ? g2 - groups : g2;
  const int64_t at = w - g2 * tokens, b = at / a.l, l = at - b * a.l;
  const int64_t row = (a.starts != nullptr ? a.starts[b] : a.start) + l;
  // rows outside the table do not exist: the tokens that would go there are dropped
  if (row < 0 || row >= a.n_table * a.block) return;
  if (a.counts != nullptr && l >= a.counts[b]) return;
  const int64_t page = a.pages[b * a.n_table + row / a.block];
  if (page < 0 || page >= a.n_pages) return;
  ChunkTurn u;
  u.other = -1;
  if (!is_v) u = chunk_turn(a.turn, a.turn.table != nullptr ? table_row(a.turn, at, row) : 0, c);
  const Strides& s = is_v ? a.vs : a.ks;
  const uint16_t* x = (is_v ? a.v : a.k) + b * s.b + l * s.l;
  uint8_t* const codes = is_v ? a.v_pages : a.k_pages;
  uint8_t* const scale = is_v ? a.v_scale : a.k_scale;
  const int end = (g + 1) * per_group < a.heads ? (g + 1) * per_group : a.heads;
  for (int h = g * per_group; h < end; ++h) {
    const uint16_t* p = x + h * s.h;
    uint4 own = *reinterpret_cast<const uint4*>(p + 8 * c);
    if (u.other >= 0) {
      const uint4 other = INTERLEAVED ? own : *reinterpret_cast<const uint4*>(p + u.other);
      own = turned(u, own, other, INTERLEAVED);
    }
    float y[8], amax = 0.f;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = bf16_at(own, e);
      const float m = fabsf(y[e]);
      if (m < INFINITY) amax = fmaxf(amax, m);
      bad |= y[e] != y[e];
    }
    amax = fmaxf(amax, __shfl_xor(amax, 1));
    amax = fmaxf(amax, __shfl_xor(amax, 2));
    const uint64_t any = __builtin_amdgcn_ballot_w64(bad) >> (threadIdx.x % 64 & ~3);
    // amax = m 2^x with 1/2 <= m < 1, and 6 = 3/4 2^3
    int e = kPagedExpMin;
    if (amax > 0.f) {
      e = __builtin_amdgcn_frexp_expf(amax) - (__builtin_amdgcn_frexp_mantf(amax) <= 0.75f ? 3 : 2);
      e = e < kPagedExpMin ? kPagedExpMin : (e > kPagedExpMax ? kPagedExpMax : e);
    }
    const float inv = __builtin_amdgcn_ldexpf(1.f, -e);
    // (the conversion rounds to the nearest, ties to even, and saturates)
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[0] * inv, y[1] * inv, 1.f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[2] * inv, y[3] * inv, 1.f, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[4] * inv, y[5] * inv, 1.f, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[6] * inv, y[7] * inv, 1.f, 3);
    const int64_t at_row = (page * a.heads + h) * a.block + row % a.block;
    *reinterpret_cast<uint32_t*>(codes + at_row * (a.d / 2) + 4 * c) = r;
    if (c % 4 == 0) scale[at_row * (a.d / 32) + c / 4] = (uint8_t)((any & 15) != 0 ? kPagedNan : e + 127);
  }
}

// One thread per 8 codes.
__global__ __launch_bounds__(256) void paged_read_kernel(PagedArgs a) {
  const int cpr = a.d / 8;
  const int64_t per_b = (int64_t)a.heads * a.l * cpr, n = a.b * per_b;
  int64_t i = group_of_rows() * 256 + threadIdx.x;
  // the first n threads take K where it is wanted, the next n (or the first) V
  const bool is_v = a.k_out == nullptr || i >= n;
  if (a.k_out != nullptr && is_v) i -= n;
  if (i >= n || (is_v && a.v_out == nullptr)) return;
  const int64_t b = i / per_b, r = i - b * per_b, w = r / cpr, h = w / a.l, row = a.start + w - h * a.l;
  const int c = (int)(r - w * cpr);
  const int64_t page = a.pages[b * a.n_table + row / a.block];
  uint4 out = make_uint4(0, 0, 0, 0);
  if (page >= 0 && page < a.n_pages) {
    const int64_t at_row = (page * a.heads + h) * a.block + row % a.block;
    const uint32_t u = *reinterpret_cast<const uint32_t*>((is_v ? a.v_pages : a.k_pages) + at_row * (a.d / 2) + 4 * c);
    const float sc = __uint_as_float((uint32_t)(is_v ? a.v_scale : a.k_scale)[at_row * (a.d / 32) + c / 4] << 23);
    out.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, sc, 0));
    out.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, sc, 1));
    out.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, sc, 2));
    out.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, sc, 3));
  }
  *reinterpret_cast<uint4*>((is_v ? a.v_out : a.k_out) + 8 * i) = out;
}

hipError_t launch_paged_write(const PagedArgs& a, hipStream_t stream) {
  const int per = 1, groups = (a.heads + per - 1) / per;
  const int64_t threads = 2 * (int64_t)a.b * a.l * groups * (a.d / 8);
  const dim3 grid = rows_of_groups((threads + 255) / 256);
  if (a.turn.interleaved) paged_write_kernel<true><<<grid, 256, 0, stream>>>(a, groups, per);
  else paged_write_kernel<false><<<grid, 256, 0, stream>>>(a, groups, per);
  return hipGetLastError();
}

hipError_t launch_paged_read(const PagedArgs& a, hipStream_t stream) {
  const int64_t n = (int64_t)a.b * a.heads * a.l * (a.d / 8) * ((a.k_out != nullptr) + (a.v_out != nullptr));
  paged_read_kernel<<<rows_of_groups((n + 255) / 256), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace sparstar
