// Rotary positions (rope.hip) and the paged 4-bit key/value cache (paged.hip,
// paged_attn.hip): what the host layer hands the kernels.  Everything here is validated
// by the host layer first.
#pragma once

#include "launch.h"

namespace sparstar {

constexpr int kRopeMaxPairs = 64, kRopeMaxAxes = 4;

struct RopeTableArgs {
  const int32_t* coords;  // [rows, axes]
  float* table;           // [rows, pairs, 2]
  int64_t rows;
  int axes, pairs;
  double amplitude;
  double quarters[kRopeMaxPairs];  // freq 2 / pi: quarter turns per step
  uint8_t axis[kRopeMaxPairs];
};

// Elements between batch elements, heads and tokens.
struct Strides {
  int64_t b, h, l;
};

// The turn of a token's channels: table rows [table_rows, pairs, 2], pairs a multiple of 8.
struct Turn {
  const float* table;        // null: none
  const int32_t* positions;  // [B, L] or null: the token's row
  int64_t table_rows;
  int pairs, interleaved, back;
};

struct RopeArgs {
  const uint16_t* x;
  uint16_t* y;
  Strides xs, ys;
  Turn turn;
  int64_t l, start;
  int b, heads, d;
};

// A cache of pages: codes [n_pages, H, block, D / 2], scale bytes e + 127 [n_pages, H, block,
// D / 32], value = code * 2^e.  The exponents' range keeps every value a normal bf16 number:
// the smallest code is 1/2, the largest 6.
constexpr int kPagedExpMin = -125, kPagedExpMax = 125;
constexpr int kPagedNan = 255;  // scale byte of 32 channels with a NaN among them

struct PagedArgs {
  uint8_t *k_pages, *v_pages, *k_scale, *v_scale;
  const int32_t* pages;            // [B, n_table]
  int64_t n_table, n_pages;
  int64_t l, start;
  int b, heads, d, block;
  // writes
  const uint16_t *k, *v;
  Strides ks, vs;
  const int32_t *starts, *counts;  // [B] or null: first row and number of the new tokens
  Turn turn;                       // of k
  // reads
  uint16_t *k_out, *v_out;         // [B, H, L, D] bf16, either may be null
};

// Attention over the pages: as over the 8-bit cache, whose `cap` is not used.
struct PagedAttnArgs : CacheAttnArgs {
  const int32_t* pages;            // [B, n_table]
  int64_t n_table, n_pages;
  float* part32;                   // part_o, which holds fp32 here: unnormalised P V
  int waves, token_waves;          // of a work-group (launcher only), as in PagedPlan
  int join_groups;                 // (launcher only, more than 32 rows)
};

// Work-groups are launched in rows of at most 2^20: a launch may have fewer than 2^32 threads
// along each axis.  (The last row's may be more than there is work for.)
inline dim3 rows_of_groups(int64_t n) {
  constexpr int64_t kRow = 1 << 20;
  const int64_t rows = (n + kRow - 1) / kRow;
  return dim3((uint32_t)((n + rows - 1) / rows), (uint32_t)rows);
}

// What work-group w of a read has to do: the first n take K where it is wanted, the next n (or
// the first) V where that is, and those that only fill the last row of the grid nothing.
struct ReadGroup {
  int64_t at;
  bool is_v, any;
};
constexpr ReadGroup read_group(int64_t w, int64_t n, bool want_k, bool want_v) {
  const bool is_v = !want_k || w >= n;
  return ReadGroup{want_k && is_v ? w - n : w, is_v, w < n * (int(want_k) + int(want_v))};
}

hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t stream);
hipError_t launch_rope(const RopeArgs& a, hipStream_t stream);
hipError_t launch_paged_write(const PagedArgs& a, hipStream_t stream);
hipError_t launch_paged_read(const PagedArgs& a, hipStream_t stream);
hipError_t launch_paged_attn(const PagedAttnArgs& a, int d, bool dense, hipStream_t stream);

}  // namespace sparstar
