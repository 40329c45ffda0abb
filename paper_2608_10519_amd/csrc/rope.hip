// Rotary positions: the table of cosines and sines, and the turn of queries and keys.
#include "rope_device.h"

namespace sparstar {

// One thread per pair and N rows, of which a work-group takes 256 / pairs at a time.  16 rows a
// thread read their coordinates side by side: 144,512 rows of 64 pairs 15.2 us (4.9 TB/s, all of
// it writes), 27.1 with one row; with fewer than 8,192 work-groups of one row a thread those start
// and end sooner (32,768 rows 7.5 and 6.5 us, 16,384 the same).
//
// The angle is taken in quarter turns, in fp64.  Adding 1.5 * 2^52 rounds it to a whole number n,
// whose last bits are the sum's last bits, and leaves r in [-1/2, 1/2]: exact, so that a far
// position keeps its fraction of a turn (|n| < 2^51, which the limits of coordinates and
// frequencies keep).  Sine and cosine of r quarter turns are their Taylor series to x^13 and
// x^14, off by less than 2^-45.
template <int N>
__global__ __launch_bounds__(256) void rope_table_kernel(RopeTableArgs a) {
  const int rpp = 256 / a.pairs;  // rows at a time
  const int row = threadIdx.x / a.pairs, p = threadIdx.x - row * a.pairs;
  if (row >= rpp) return;
  const int64_t t0 = group_of_rows() * (N * rpp) + row;
  const int32_t* coord = a.coords + t0 * a.axes + a.axis[p];
  const double per = a.quarters[p];
  const int left = a.rows - t0 < N * rpp ? (int)(a.rows - t0) : N * rpp;
  int32_t at[N];
#pragma unroll
  for (int i = 0; i < N; ++i, coord += rpp * a.axes) at[i] = i * rpp < left ? *coord : 0;
  f32x2* out = reinterpret_cast<f32x2*>(a.table) + t0 * a.pairs + p;
#pragma unroll
  for (int i = 0; i < N; ++i, out += rpp * a.pairs) {
    if (i * rpp >= left) return;
    const double x = per * at[i], w = x + 6755399441055744.0, r = x - (w - 6755399441055744.0), z = r * r;
    const uint32_t n = (uint32_t)__builtin_bit_cast(uint64_t, w);
    // (pi/2)^k / k!
    double s = 5.692172921967924e-08;
    s = fma(s, z, -3.598843235212084e-06);
    s = fma(s, z, 1.6044118478735982e-04);
    s = fma(s, z, -4.681754135318688e-03);
    s = fma(s, z, 7.969262624616704e-02);
    s = fma(s, z, -6.459640975062462e-01);
    s = fma(s, z, 1.5707963267948966);
    double c = -6.386603083791849e-09;
    c = fma(c, z, 4.710874778818169e-07);
    c = fma(c, z, -2.5202042373060605e-05);
    c = fma(c, z, 9.1926027483942658e-04);
    c = fma(c, z, -2.086348076335296e-02);
    c = fma(c, z, 2.5366950790104802e-01);
    c = fma(c, z, -1.2337005501361698);
    c = fma(c, z, 1.0);
    const float cf = (float)(c * a.amplitude), sf = (float)(s * (r * a.amplitude));
    const float cq = n & 1 ? sf : cf, sq = n & 1 ? cf : sf;
    const f32x2 cs = {__uint_as_float(__float_as_uint(cq) ^ ((n + 1) << 30 & 0x80000000u)),
                      __uint_as_float(__float_as_uint(sq) ^ (n << 30 & 0x80000000u))};
    __builtin_nontemporal_store(cs, out);
  }
}

// One thread per (token, chunk of 8 channels) and N heads, whose rows are loaded before the
// first is turned: the table's entries (64 bytes a thread, against 48 for the chunk, its
// partners' and its result) are read and made fp64 once.  A row lies in one wave, whose loads
// of all of it come before its stores: y may be x.
//
// Memory bounds it.  24 heads, D = 128: 11,520 rows 29.5 us with three heads a thread (5.0 TB/s),
// 34.9 with one, 29.8 with two, 29.2 with four; 72,000 rows 176 us (5.2 TB/s), 252, 189 and 173;
// 3,000 rows 7.7 us, 9.7, 8.3 and 8.0.  Below some 8,192 rows of all heads three heads a thread
// leave CUs without work: 340 rows 3.3 us with one and 3.1 with three, 170 2.8 and 3.0, 64 2.4
// and 2.9 (in a captured graph, without the calls' own time).  Results go past
// the L2's share of what is read (11,520 rows 33 us without).
template <bool INTERLEAVED, int N>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a) {
  const TokenChunk t = token_chunk((int64_t)a.b * a.l, a.l, a.d == 128 ? 4 : 3);
  if (!t.ok) return;
  const ChunkTurn u = chunk_turn(a.turn, table_row(a.turn, t.at, a.start + t.l), t.c);
  const uint16_t* x = a.x + t.b * a.xs.b + t.l * a.xs.l + t.group * N * a.xs.h;
  uint16_t* y = a.y + t.b * a.ys.b + t.l * a.ys.l + t.group * N * a.ys.h + 8 * t.c;
  const int left = a.heads - (int)t.group * N;  // heads
  uint4 own[N], other[N];
#pragma unroll
  for (int h = 0; h < N; ++h) {
    if (h >= left) continue;
    own[h] = *reinterpret_cast<const uint4*>(x + h * a.xs.h + 8 * t.c);
    if (!INTERLEAVED && u.other >= 0) other[h] = *reinterpret_cast<const uint4*>(x + h * a.xs.h + u.other);
  }
#pragma unroll
  for (int h = 0; h < N; ++h) {
    if (h >= left) continue;
    const uint4 r = u.other >= 0 ? turned(u, own[h], INTERLEAVED ? own[h] : other[h], INTERLEAVED) : own[h];
    store_once(y + h * a.ys.h, r);
  }
}

hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t stream) {
  const int rpp = 256 / a.pairs;
  if (a.rows >= 8192 * rpp) rope_table_kernel<16><<<rows_of_groups((a.rows + 16 * rpp - 1) / (16 * rpp)), 256, 0, stream>>>(a);
  else rope_table_kernel<1><<<rows_of_groups((a.rows + rpp - 1) / rpp), 256, 0, stream>>>(a);
  return hipGetLastError();
}

template <int N>
static hipError_t launch_turns(const RopeArgs& a, hipStream_t stream) {
  const dim3 grid = token_grid((a.heads + N - 1) / N, (int64_t)a.b * a.l, a.d);
  if (a.turn.interleaved) rope_kernel<true, N><<<grid, 256, 0, stream>>>(a);
  else rope_kernel<false, N><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t stream) {
  return (int64_t)a.b * a.heads * a.l >= 8192 ? launch_turns<3>(a, stream) : launch_turns<1>(a, stream);
}

}  // namespace sparstar
