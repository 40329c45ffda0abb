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

// The largest magnitude of a group of four threads' values, as bf16 bits, by each of them.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t group_max(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 15, 15, true));  // lanes 1 0 3 2
  return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 15, 15, true));  // lanes 2 3 0 1
}

// Scale byte of the 32 channels that this thread and its three neighbours hold.
__device__ __forceinline__ uint32_t scale_byte_of(uint4 w) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
  u16x2 big = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) big = __builtin_elementwise_max(big, __builtin_bit_cast(u16x2, u[i] & 0x7fff7fffu));
  uint32_t m = group_max(max(big[0], big[1]));
  bool nan = false;
  if (m >= 0x7f80) {  // not finite (the same in all four): the largest of what is
    uint32_t top = 0;
    m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t x = (i % 2 ? u[i / 2] >> 16 : u[i / 2]) & 0x7fff;
      top = max(top, x);
      if (x < 0x7f80) m = max(m, x);
    }
    nan = group_max(top) > 0x7f80;
    m = group_max(m);
  }
  // m = 1.f 2^(E - 127) with E and the 7 bits f its fields: e is E - 127 - 2, and one more where
  // 1.f > 3/2, 6 being 3/2 2^2
  const int byte = (int)((m + 63) >> 7) - 2;
  return nan ? kPagedNan : (uint32_t)min(max(byte, kPagedExpMin + 127), kPagedExpMax + 127);
}

// A 4 x 4 transposition among four neighbouring threads: thread i gets every thread's w[i], by
// two exchanges of the half that the other needs.
__device__ __forceinline__ uint4 transposed(const uint32_t (&w)[4], int i) {
  auto from = [](uint32_t x, auto perm) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, perm(), 15, 15, true);
  };
  auto next = [] { return 0xb1; };    // lanes 1 0 3 2
  auto second = [] { return 0x4e; };  // lanes 2 3 0 1
  const bool odd = i & 1, high = i & 2;
  const uint32_t a = from(odd ? w[0] : w[1], next), b = from(odd ? w[2] : w[3], next);
  const uint2 lo = odd ? make_uint2(a, w[1]) : make_uint2(w[0], a);  // this pair's of i % 2
  const uint2 hi = odd ? make_uint2(b, w[3]) : make_uint2(w[2], b);  // and of i % 2 + 2
  const uint2 give = high ? lo : hi;
  const uint2 got = make_uint2(from(give.x, second), from(give.y, second));
  return high ? make_uint4(got.x, got.y, hi.x, hi.y) : make_uint4(lo.x, lo.y, got.x, got.y);
}

// One thread per (K or V, token, chunk of 8 channels) and N heads, as rope_kernel; four
// neighbouring threads share a scale.  With four heads each of the four stores one head's codes
// and scale, 16 bytes in place of four.
//
// 24 heads, D = 128, keys rotated: 11,520 tokens 42 us (4.4 TB/s), 64 with one head a thread;
// 72,000 tokens 232 us (5.0 TB/s), 386; 500 tokens 5.2 and 5.5, 340 4.0 both, 170 3.9 and 3.6 (in
// a captured graph).  Three heads a thread, each storing its own codes: 43 and 247.  Unrotated 36 and 208: K's rotation in fp64 is what memory does not hide.  Stores past
// the caches write 11,520 tokens in 39 us, but a read of them takes 44 then, 27 now.
template <bool INTERLEAVED, int N>
__global__ __launch_bounds__(256) void paged_write_kernel(PagedArgs a) {
  static_assert(N == 1 || N == 4);
  const TokenChunk t = token_chunk((int64_t)a.b * a.l, a.l, a.d == 128 ? 4 : 3);
  if (!t.ok) return;  // (whole rows of threads: whole groups of four)
  // (K and V in turn: the turns' work lies beside V's loads)
  const bool is_v = t.group % 2 != 0;
  const int h0 = (int)(t.group / 2) * N, left = a.heads - h0, c = t.c;
  const int64_t row = (a.starts != nullptr ? a.starts[t.b] : a.start) + t.l;
  const int block_bits = a.block == 128 ? 7 : 6;
  // rows outside the table do not exist: the tokens that would go there are dropped
  if (row < 0 || row >= a.n_table << block_bits) return;
  if (a.counts != nullptr && t.l >= a.counts[t.b]) return;
  const int64_t page = a.pages[t.b * a.n_table + (row >> block_bits)];
  if (page < 0 || page >= a.n_pages) return;
  ChunkTurn u;
  u.other = -1;
  if (!is_v && a.turn.table != nullptr) u = chunk_turn(a.turn, table_row(a.turn, t.at, row), c);
  const Strides& s = is_v ? a.vs : a.ks;
  const uint16_t* x = (is_v ? a.v : a.k) + t.b * s.b + t.l * s.l + h0 * s.h;
  const int64_t at_row = ((page * a.heads + h0) << block_bits) + (row & (a.block - 1));
  uint8_t* const codes = (is_v ? a.v_pages : a.k_pages) + at_row * (a.d / 2);
  uint8_t* const scale = (is_v ? a.v_scale : a.k_scale) + at_row * (a.d / 32) + c / 4;
  uint4 own[N], other[N];
#pragma unroll
  for (int h = 0; h < N; ++h) {
    if (h >= left) continue;
    own[h] = *reinterpret_cast<const uint4*>(x + h * s.h + 8 * c);
    if (!INTERLEAVED && u.other >= 0) other[h] = *reinterpret_cast<const uint4*>(x + h * s.h + u.other);
  }
  uint32_t code[N], byte[N];
#pragma unroll
  for (int h = 0; h < N; ++h) {
    code[h] = byte[h] = 0;
    if (h >= left) continue;
    const uint4 w = u.other >= 0 ? turned(u, own[h], INTERLEAVED ? own[h] : other[h], INTERLEAVED) : own[h];
    byte[h] = scale_byte_of(w);
    // (the conversion divides by the scale, rounds to the nearest, ties to even, and saturates)
    const float sc = __uint_as_float(byte[h] << 23);
    code[h] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code[h], __builtin_bit_cast(bf16x2, w.x), sc, 0);
    code[h] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code[h], __builtin_bit_cast(bf16x2, w.y), sc, 1);
    code[h] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code[h], __builtin_bit_cast(bf16x2, w.z), sc, 2);
    code[h] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code[h], __builtin_bit_cast(bf16x2, w.w), sc, 3);
  }
  if constexpr (N == 4) {
    const int h = c % 4;
    const uint4 w = transposed(code, h);
    if (h >= left) return;
    *reinterpret_cast<uint4*>(codes + h * (a.block * (a.d / 2)) + 16 * (c / 4)) = w;
    scale[h * (a.block * (a.d / 32))] = (uint8_t)(h == 0 ? byte[0] : h == 1 ? byte[1] : h == 2 ? byte[2] : byte[3]);
  } else {
    *reinterpret_cast<uint32_t*>(codes + 4 * c) = code[0];
    if (c % 4 == 0) *scale = (uint8_t)byte[0];
  }
}

// One work-group per (K or V, batch * head, P times 256 / TPR rows), TPR threads a row with W
// times 8 channels each.
template <int CPR, int W, int P, bool ONCE>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedArgs a) {
  constexpr int TPR = CPR / W, RPP = 256 / TPR;
  const int64_t per = (a.l + RPP * P - 1) / (RPP * P), n = (int64_t)a.b * a.heads * per;
  const ReadGroup group = read_group(group_of_rows(), n, a.k_out != nullptr, a.v_out != nullptr);
  if (!group.any) return;
  const bool is_v = group.is_v;
  const int64_t w = group.at;
  const int64_t bh = divide(w, per), b = divide(bh, a.heads), h = bh - b * a.heads;
  const int64_t l0 = (w - bh * per) * (RPP * P) + threadIdx.x / TPR;
  const int c = threadIdx.x % TPR, block_bits = a.block == 128 ? 7 : 6;
  const uint8_t* const codes = is_v ? a.v_pages : a.k_pages;
  const uint8_t* const scale = is_v ? a.v_scale : a.k_scale;
  uint32_t u[P][W];
  float sc[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
#pragma unroll
    for (int k = 0; k < W; ++k) u[i][k] = 0;
    sc[i] = 0.f;
    const int64_t l = l0 + i * RPP, row = a.start + l;
    if (l >= a.l) continue;
    const int64_t page = a.pages[b * a.n_table + (row >> block_bits)];
    if (page < 0 || page >= a.n_pages) continue;
    const int64_t at_row = ((page * a.heads + h) << block_bits) + (row & (a.block - 1));
    __builtin_memcpy(u[i], __builtin_assume_aligned(codes + at_row * (4 * CPR) + 4 * W * c, 4 * W), 4 * W);
    sc[i] = __uint_as_float((uint32_t)scale[at_row * (CPR / 4) + W * c / 4] << 23);
  }
  uint16_t* const out = (is_v ? a.v_out : a.k_out) + ((bh * a.l + l0) * TPR + c) * (8 * W);
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (l0 + i * RPP >= a.l) continue;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      uint4 r;
      r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u[i][k], sc[i], 0));
      r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u[i][k], sc[i], 1));
      r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u[i][k], sc[i], 2));
      r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u[i][k], sc[i], 3));
      uint16_t* const to = out + i * (RPP * CPR * 8) + 8 * k;
      if constexpr (ONCE) store_once(to, r);
      else *reinterpret_cast<uint4*>(to) = r;
    }
  }
}

template <int N>
static hipError_t launch_writes(const PagedArgs& a, hipStream_t stream) {
  const dim3 grid = token_grid(2 * ((a.heads + N - 1) / N), (int64_t)a.b * a.l, a.d);
  if (a.turn.interleaved) paged_write_kernel<true, N><<<grid, 256, 0, stream>>>(a);
  else paged_write_kernel<false, N><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_write(const PagedArgs& a, hipStream_t stream) {
  return (int64_t)a.b * a.heads * a.l >= 8192 ? launch_writes<4>(a, stream) : launch_writes<1>(a, stream);
}

template <int CPR, int W, int P, bool ONCE>
static hipError_t launch_reads(const PagedArgs& a, hipStream_t stream) {
  const int64_t rows = 256 / (CPR / W) * P, n = (int64_t)a.b * a.heads * ((a.l + rows - 1) / rows);
  const dim3 grid = rows_of_groups(n * ((a.k_out != nullptr) + (a.v_out != nullptr)));
  paged_read_kernel<CPR, W, P, ONCE><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

// Rows that the last-level cache holds, 256 MB, are best written past the L2 with 16 bytes a
// lane side by side: 24 heads of 11,520 rows, D = 128, K and V (141 MB) 26 us, 37 with 32
// bytes a lane through the L2; K alone 14.8 and 19.3.  Beyond it the latter is the faster:
// 72,000 rows 216 and 263 us, K alone (442 MB) 110 and 132.
template <int CPR>
static hipError_t launch_reads(const PagedArgs& a, hipStream_t stream) {
  const double bytes = 16.0 * CPR * a.b * a.heads * a.l * ((a.k_out != nullptr) + (a.v_out != nullptr));
  return bytes <= 192e6 ? launch_reads<CPR, 1, 2, true>(a, stream) : launch_reads<CPR, 2, 1, false>(a, stream);
}

hipError_t launch_paged_read(const PagedArgs& a, hipStream_t stream) {
  return a.d == 128 ? launch_reads<16>(a, stream) : launch_reads<8>(a, stream);
}

}  // namespace sparstar
