// Rotary positions: the table of cosines and sines, and the turn of queries and keys.
#include "rope_device.h"

namespace sparstar {

// One thread per (row, pair).  The angle in turns is taken in fp64 and reduced exactly (x -
// rint(x)), so that far positions keep their fraction of a turn.
__global__ __launch_bounds__(256) void rope_table_kernel(RopeTableArgs a) {
  const int64_t i = group_of_rows() * 256 + threadIdx.x;
  if (i >= a.rows * a.pairs) return;
  const int64_t t = i / a.pairs;
  const int p = (int)(i - t * a.pairs);
  const double turns = a.turns[p] * a.coords[t * a.axes + a.axis[p]];
  double s, c;
  sincospi(2.0 * (turns - rint(turns)), &s, &c);
  reinterpret_cast<float2*>(a.table)[i] = make_float2((float)(a.amplitude * c), (float)(a.amplitude * s));
}

// One thread per (token, chunk of 8 channels), for a group of heads: the table's entries are
// read and made fp64 once.  A row lies in one wave, whose loads of all of it come before its
// stores: y may be x.
template <bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a, int groups, int per_group) {
  const int cpr = a.d / 8;
  const int64_t i = group_of_rows() * 256 + threadIdx.x;
  const int64_t tokens = (int64_t)a.b * a.l, w = i / cpr;
  if (w >= tokens * groups) return;
  const int c = (int)(i - w * cpr);
  const int g = (int)(w / tokens);
  const int64_t at = w - g * tokens, b = at / a.l, l = at - b * a.l;
  const ChunkTurn u = chunk_turn(a.turn, table_row(a.turn, at, a.start + l), c);
  const uint16_t* x = a.x + b * a.xs.b + l * a.xs.l;
  uint16_t* y = a.y + b * a.ys.b + l * a.ys.l + 8 * c;
  const int end = (g + 1) * per_group < a.heads ? (g + 1) * per_group : a.heads;
  for (int h = g * per_group; h < end; ++h) {
    const uint16_t* row = x + h * a.xs.h;
    const uint4 own = *reinterpret_cast<const uint4*>(row + 8 * c);
    uint4 r = own;
    if (u.other >= 0) {
      const uint4 other = INTERLEAVED ? own : *reinterpret_cast<const uint4*>(row + u.other);
      r = turned(u, own, other, INTERLEAVED);
    }
    *reinterpret_cast<uint4*>(y + h * a.ys.h) = r;
  }
}

hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t stream) {
  rope_table_kernel<<<rows_of_groups((a.rows * a.pairs + 255) / 256), 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t stream) {
  const int per = 1, groups = (a.heads + per - 1) / per;
  const int64_t threads = (int64_t)a.b * a.l * groups * (a.d / 8);
  const dim3 grid = rows_of_groups((threads + 255) / 256);
  if (a.turn.interleaved) rope_kernel<true><<<grid, 256, 0, stream>>>(a, groups, per);
  else rope_kernel<false><<<grid, 256, 0, stream>>>(a, groups, per);
  return hipGetLastError();
}

}  // namespace sparstar
