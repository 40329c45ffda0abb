// C ABI of the rotary positions: host-side validation and launches.  As in host_api.cpp,
// every argument is checked before the first HIP call.
#include <math.h>
#include <stdio.h>

#include <algorithm>

#include "rope_check.h"

using namespace sparstar;

namespace sparstar {

int check_strides(sparstar_strides s, int B, int H, int64_t L, int D, bool output, const char* name, Strides* out) {
  char msg[160];
  auto refuse = [&](const char* why) {
    snprintf(msg, sizeof msg, "%s: %s", name, why);
    return report_error(SPARSTAR_ERR_INVALID_ARG, msg);
  };
  struct Dim {
    int64_t stride, size;
  } d[3] = {{B > 1 ? s.batch : 0, B}, {H > 1 ? s.head : 0, H}, {L > 1 ? s.token : 0, L}};
  *out = Strides{d[0].stride, d[1].stride, d[2].stride};
  int64_t reach = D;
  for (const Dim& x : d) {
    if (x.stride < 0 || x.stride % 8 != 0) return refuse("strides must be multiples of 8 elements, not negative");
    if (x.stride > (int64_t(1) << 46)) return refuse("strides too large");
    if (x.size > 1 && x.stride > ((int64_t(1) << 46) - reach) / (x.size - 1)) return refuse("tensor too large");
    if (x.size > 1) reach += x.stride * (x.size - 1);
  }
  if (!output || L == 0) return SPARSTAR_OK;  // (no rows that could overlap)
  std::sort(d, d + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  int64_t within = D;  // elements from the first to the last of the dimensions so far
  for (const Dim& x : d) {
    if (x.size <= 1) continue;
    if (x.stride < within) return refuse("the rows of an output may not overlap");
    within += x.stride * (x.size - 1);
  }
  return SPARSTAR_OK;
}

int check_turn(const float* table, int64_t table_rows, int pairs, int interleaved, const int32_t* positions, int D,
               int64_t start, int64_t L, bool anywhere, Turn* out) {
  if (pairs < 8 || pairs % 8 != 0 || pairs > D / 2)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "pairs must be a multiple of 8 in [8, D / 2]");
  if (table_rows < (L > 0) || table_rows > (int64_t(1) << 40))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "table_rows must be in [1, 2^40], or 0 without tokens");
  if (reinterpret_cast<uintptr_t>(table) & 15u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "the table must be 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(positions) & 3u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "positions must be 4-byte aligned");
  if (!positions && !anywhere && (start < 0 || start > table_rows || L > table_rows - start))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "the positions [start, start + L) must lie inside the table");
  *out = Turn{table, positions, table_rows, pairs, interleaved != 0, 0};
  return SPARSTAR_OK;
}

}  // namespace sparstar

extern "C" int sparstar_rope_frequencies(int pairs, double base, double factor, double length, double slow, double fast,
                                         double* out) {
  if (pairs < 1) return report_error(SPARSTAR_ERR_INVALID_ARG, "pairs must be >= 1");
  if (!out) return report_error(SPARSTAR_ERR_INVALID_ARG, "out must be non-null");
  if (!(base > 1.0) || isinf(base)) return report_error(SPARSTAR_ERR_INVALID_ARG, "base must be > 1 and finite");
  if (!(factor >= 1.0) || isinf(factor)) return report_error(SPARSTAR_ERR_INVALID_ARG, "factor must be >= 1 and finite");
  if (factor != 1.0 && (!(length > 0.0) || isinf(length) || !(slow >= 0.0) || !(fast > slow) || isinf(fast)))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "length must be > 0 and 0 <= slow < fast");
  for (int p = 0; p < pairs; ++p) {
    const double f = pow(base, -double(p) / pairs);
    double keep = 1.0;
    if (factor != 1.0)
      keep = fmin(1.0, fmax(0.0, (length * f / 6.283185307179586477 - slow) / (fast - slow)));
    out[p] = f * (keep + (1.0 - keep) / factor);
  }
  return clear_error();
}

extern "C" int sparstar_rope_table(const int32_t* coords, int64_t rows, int axes, int pairs, const double* freq,
                                   const int32_t* axis, double amplitude, float* table, void* stream) {
  if (rows < 0 || rows > (int64_t(1) << 40)) return report_error(SPARSTAR_ERR_INVALID_ARG, "rows must be in [0, 2^40]");
  if (axes < 1 || axes > kRopeMaxAxes) return report_error(SPARSTAR_ERR_INVALID_ARG, "axes must be in [1, 4]");
  if (pairs < 1 || pairs > kRopeMaxPairs) return report_error(SPARSTAR_ERR_INVALID_ARG, "pairs must be in [1, 64]");
  if (!freq) return report_error(SPARSTAR_ERR_INVALID_ARG, "freq must be non-null");
  if (!isfinite(amplitude)) return report_error(SPARSTAR_ERR_INVALID_ARG, "amplitude must be finite");
  RopeTableArgs a{};
  for (int p = 0; p < pairs; ++p) {
    if (!(fabs(freq[p]) <= 1048576.0))
      return report_error(SPARSTAR_ERR_INVALID_ARG, "frequencies must be finite, of at most 2^20");
    const int32_t x = axis ? axis[p] : 0;
    if (x < 0 || x >= axes) return report_error(SPARSTAR_ERR_INVALID_ARG, "a pair's axis must be in [0, axes)");
    a.quarters[p] = freq[p] / 1.570796326794896619;
    a.axis[p] = uint8_t(x);
  }
  if (rows > 0 && (!coords || !table))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "coords and table must be non-null");
  if ((reinterpret_cast<uintptr_t>(coords) & 3u) || (reinterpret_cast<uintptr_t>(table) & 7u))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "coords must be 4-byte, the table 8-byte aligned");
  if (rows == 0) return clear_error();
  a.coords = coords;
  a.table = table;
  a.rows = rows;
  a.axes = axes;
  a.pairs = pairs;
  a.amplitude = amplitude;
  const hipError_t e = launch_rope_table(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return report_error(SPARSTAR_ERR_HIP, hipGetErrorString(e));
  return clear_error();
}

static int rope_common(const void* x, sparstar_strides xs, int B, int H, int64_t L, int D, const float* table,
                       int64_t table_rows, int pairs, int interleaved, const int32_t* positions, int64_t start,
                       void* y, sparstar_strides ys, void* stream, bool back) {
  if (int rc = check_attn_sizes(B, H, L, 1, D, 64)) return rc;
  RopeArgs a{};
  if (int rc = check_strides(xs, B, H, L, D, false, "x", &a.xs)) return rc;
  if (int rc = check_strides(ys, B, H, L, D, true, "y", &a.ys)) return rc;
  if (int rc = check_turn(table, table_rows, pairs, interleaved, positions, D, start, L, false, &a.turn)) return rc;
  if (L > 0 && (!x || !y || !table)) return report_error(SPARSTAR_ERR_INVALID_ARG, "x, y and table must be non-null");
  if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y)) & 15u)
    return report_error(SPARSTAR_ERR_INVALID_ARG, "x and y must be 16-byte aligned");
  if (x && x == y && (a.xs.b != a.ys.b || a.xs.h != a.ys.h || a.xs.l != a.ys.l))
    return report_error(SPARSTAR_ERR_INVALID_ARG, "y may be x only with the same strides");
  if (L == 0) return clear_error();
  a.turn.back = back;
  a.x = static_cast<const uint16_t*>(x);
  a.y = static_cast<uint16_t*>(y);
  a.l = L;
  a.start = start;
  a.b = B;
  a.heads = H;
  a.d = D;
  const hipError_t e = launch_rope(a, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return report_error(SPARSTAR_ERR_HIP, hipGetErrorString(e));
  return clear_error();
}

extern "C" int sparstar_rope_fwd(const void* x, sparstar_strides xs, int B, int H, int64_t L, int D,
                                 const float* table, int64_t table_rows, int pairs, int interleaved,
                                 const int32_t* positions, int64_t start, void* y, sparstar_strides ys, void* stream) {
  return rope_common(x, xs, B, H, L, D, table, table_rows, pairs, interleaved, positions, start, y, ys, stream, false);
}

extern "C" int sparstar_rope_bwd(const void* dy, sparstar_strides dys, int B, int H, int64_t L, int D,
                                 const float* table, int64_t table_rows, int pairs, int interleaved,
                                 const int32_t* positions, int64_t start, void* dx, sparstar_strides dxs,
                                 void* stream) {
  return rope_common(dy, dys, B, H, L, D, table, table_rows, pairs, interleaved, positions, start, dx, dxs, stream,
                     true);
}
