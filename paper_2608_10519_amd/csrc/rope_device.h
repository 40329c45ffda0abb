// The turn of a row's channels by its position, for the kernels that rotate (rope.hip) and
// that rotate on the way into the cache (paged.hip).
//
// A thread has 8 neighbouring channels (a chunk) of a row.  Each of their results is
// own * ct + other * st, the other channel of the pair coming from the chunk itself
// (interleaved) or from one pairs channels away.  A bf16 value times an fp32 entry of the
// table has 32 significant bits: exact in fp64, so that the sum alone is rounded, and every
// path that rotates the same key gives the same bits, which an fp32 sum next to a border of
// the 4-bit codes would not.
#pragma once

#include "attn_device.h"
#include "paged.h"

namespace sparstar {

struct ChunkTurn {
  double ct[8], st[8];
  int other;  // channel offset of the chunk that holds the partners; negative: the row passes
};

// Table row of token i of batch element b, which lands in (or is) row `row`.
__device__ __forceinline__ int64_t table_row(const Turn& t, int64_t at, int64_t row) {
  const int64_t p = t.positions != nullptr ? t.positions[at] : row;
  return p < 0 ? 0 : (p < t.table_rows ? p : t.table_rows - 1);
}

// Chunk c of a row whose table row is r.
__device__ __forceinline__ ChunkTurn chunk_turn(const Turn& t, int64_t r, int c) {
  ChunkTurn u;
  u.other = -1;
  const int hc = t.pairs / 8;  // chunks of the pairs' first channels
  if (t.table == nullptr || c >= 2 * hc) return u;
  const float sign = t.back ? -1.f : 1.f;
  const float* const row = t.table + r * t.pairs * 2;
  if (t.interleaved) {
    const float4* p = reinterpret_cast<const float4*>(row + 8 * c);  // four pairs from 4 c on
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 w = p[i];
      u.ct[4 * i] = u.ct[4 * i + 1] = w.x;
      u.ct[4 * i + 2] = u.ct[4 * i + 3] = w.z;
      u.st[4 * i] = -sign * w.y, u.st[4 * i + 1] = sign * w.y;
      u.st[4 * i + 2] = -sign * w.w, u.st[4 * i + 3] = sign * w.w;
    }
    u.other = 8 * c;
  } else {
    const bool second = c >= hc;
    const float4* p = reinterpret_cast<const float4*>(row + 16 * (second ? c - hc : c));  // eight pairs
    const float s = second ? sign : -sign;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 w = p[i];
      u.ct[2 * i] = w.x, u.ct[2 * i + 1] = w.z;
      u.st[2 * i] = s * w.y, u.st[2 * i + 1] = s * w.w;
    }
    u.other = 8 * (second ? c - hc : c + hc);
  }
  return u;
}

__device__ __forceinline__ float bf16_at(const uint4& u, int i) {
  const uint32_t w = i < 2 ? u.x : (i < 4 ? u.y : (i < 6 ? u.z : u.w));
  return i % 2 ? bf16_hi(w) : bf16_lo(w);
}

// The chunk's results in bf16; `other` holds the partners' chunk (interleaved: `own` again).
__device__ __forceinline__ uint4 turned(const ChunkTurn& u, uint4 own, uint4 other, bool interleaved) {
  float r[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double x = interleaved ? bf16_at(other, i ^ 1) : bf16_at(other, i);
    r[i] = (float)fma(x, u.st[i], (double)bf16_at(own, i) * u.ct[i]);
  }
  return make_uint4(pack2_bf16(r[0], r[1]), pack2_bf16(r[2], r[3]), pack2_bf16(r[4], r[5]), pack2_bf16(r[6], r[7]));
}

// 16 bytes that this kernel does not read again, past the caches' share of what it does.
__device__ __forceinline__ void store_once(uint16_t* p, uint4 r) {
  __builtin_nontemporal_store((u32x4){r.x, r.y, r.z, r.w}, reinterpret_cast<u32x4*>(p));
}

__device__ __forceinline__ int64_t group_of_rows() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// a / b of numbers that mostly fit 32 bits, where a division takes a fifth of the instructions.
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// The work of a thread of a launch over (group of heads, token of any batch element, chunk):
// work-groups take 256 / cpr tokens of one group.
struct TokenChunk {
  int64_t group, at, b, l;  // at = b L + l
  int c;
  bool ok;
};
__device__ __forceinline__ TokenChunk token_chunk(int64_t tokens, int64_t len, int cpr_bits) {
  const int tpg = 256 >> cpr_bits;
  const int64_t per_group = (tokens + tpg - 1) / tpg, w = group_of_rows();
  TokenChunk t;
  t.group = divide(w, per_group);
  t.at = (w - t.group * per_group) * tpg + (threadIdx.x >> cpr_bits);
  t.c = threadIdx.x & ((1 << cpr_bits) - 1);
  t.ok = t.at < tokens;
  t.b = tokens == len ? 0 : divide(t.at, len);
  t.l = t.at - t.b * len;
  return t;
}
inline dim3 token_grid(int64_t groups, int64_t tokens, int d) {
  const int tpg = 256 / (d / 8);
  return rows_of_groups(groups * ((tokens + tpg - 1) / tpg));
}

}  // namespace sparstar
