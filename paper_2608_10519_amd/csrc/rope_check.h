// Checks of strides and turns, which the rotations and the paged cache's writes share.
#pragma once

#include "../../include/sparstar.h"
#include "host_internal.h"
#include "paged.h"

namespace sparstar {

// The strides of a [B, H, L, D] tensor, those of a size of 1 as zero.
int check_strides(sparstar_strides s, int B, int H, int64_t L, int D, bool output, const char* name, Strides* out);

// A table and what is read of it: rows [start, start + L) where neither positions nor
// `anywhere` (first rows that only the device knows) are given.
int check_turn(const float* table, int64_t table_rows, int pairs, int interleaved, const int32_t* positions, int D,
               int64_t start, int64_t L, bool anywhere, Turn* out);

}  // namespace sparstar
