// Attention of more than 32 query rows over a cache of codes, and the join of partial
// results: shared by the 8-bit cache (cache_attn.hip) and the pages of 4-bit codes
// (paged_attn.hip).
#pragma once

#include "attn_device.h"
#include "cache_plan.h"
#include "paged.h"

namespace sparstar {

template <int D>
struct CacheCfg {
  static constexpr int KB = attn_tile_keys(D);    // keys per tile
  static constexpr int KT = KB / 32;              // 32-key sub-tiles
  static constexpr int DS = D / 16, DT = D / 32;  // 16-column steps of a row, 32-row tiles of O^T
  static constexpr int RB = D;                    // bytes per row of codes
  static constexpr int CPR = D / 16;              // 16-byte chunks per row of codes
  static constexpr int RPD = 1024 / RB;           // rows per direct-to-LDS wave load
  static constexpr int TILE = KB * RB;            // bytes of codes per tile: 4 KB
  static_assert(TILE == 4096, "4 KB tiles");
};

// eight codes -> eight bf16 values times the scale (exact)
__device__ __forceinline__ bf16x8 decode8(uint2 u, float scale) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.x, scale, false));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.x, scale, true));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.y, scale, false));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.y, scale, true));
  return __builtin_bit_cast(bf16x8, r);
}

typedef float f32x8 __attribute__((ext_vector_type(8)));

// The two kinds of cache.  A lane takes 16 codes of a tile at a time (a piece), and turns
// them into two chunks of eight bf16 values.
//
// 8 bits: e4m3 codes [BH, cap, D], a scale byte per block.
struct Codes8 {
  using Args = CacheAttnArgs;
  using Part = f16x8;  // of a range's P V (store_rows)
  static constexpr bool PAGED = false;
  struct Piece {
    uint4 u;
  };
};

// 4 bits: e2m1 codes in pages of a block, [n_pages, H, block, D / 2], a scale byte per row and
// 32 channels.
struct Codes4 {
  using Args = PagedAttnArgs;
  using Part = f32x8;
  static constexpr bool PAGED = true;
  struct Piece {
    uint2 u;
    uint32_t s;
  };
};

// eight 4-bit codes -> eight bf16 values times the scale (exact)
__device__ __forceinline__ bf16x8 decode8_4bit(uint32_t u, float scale) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 0));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 1));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 2));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, 3));
  return __builtin_bit_cast(bf16x8, r);
}

// Writes the lane's query row (its columns 32 t + 8 g + 4 h + 0..3): O and lse, or, with
// several ranges, the range's unnormalised P V with the running max (log2 units) and the two
// row sums.  m, l and le are the row's; l == 0 means no key was seen (a NaN passes on).
//
// The 8-bit cache's P V goes out in fp16, with the exponent of its scale: this rounds once more,
// by at most 2^-11 of the value, an eighth of what P's rounding to bf16 may change, for half the
// bytes of fp32.  The scale, a power of two, brings the row's largest magnitude to [2^14, 2^15),
// the top of fp16's range, so that a column down to 2^-28 of it keeps all 11 bits.  Over pages
// every 32 channels of a value have a scale of their own, so that columns may lie further apart
// than that (and than 2^-39, where nothing would be left of the smaller ones): their P V stays
// in fp32.
template <int D, class F>
__device__ __forceinline__ void store_rows(const typename F::Args& a, int64_t bh, int64_t row, int range,
                                           const f32x16 (&acc)[D / 32], float m, float l, float le, int hh) {
  float amax = 0.f;
  if (!F::PAGED && a.ranges > 1) {
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) amax = fmaxf(amax, fabsf(acc[t][e]));
    amax = half_swap_max(amax);
  }
  if (row >= a.lq) return;
  const int64_t at = bh * a.lq + row;
  if (a.ranges > 1) {
    const int64_t prow = (int64_t)range * a.bh * a.lq + at;
    int ex = 0;
    if constexpr (F::PAGED) {
      float* out = reinterpret_cast<float*>(a.part_o) + prow * D + 4 * hh;
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<float4*>(out + 32 * t + 8 * g) =
              make_float4(acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]);
    } else {
      if (amax > 0.f && amax <= 3.402823466e38f) ex = __builtin_amdgcn_frexp_expf(amax) - 15;
      ex = ex < -126 ? -126 : ex;
      const float sc = __builtin_amdgcn_ldexpf(1.0f, -ex);
      _Float16* out = reinterpret_cast<_Float16*>(a.part_o) + prow * D + 4 * hh;
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          f16x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = (_Float16)(acc[t][4 * g + e] * sc);
          *reinterpret_cast<f16x4*>(out + 32 * t + 8 * g) = w;
        }
    }
    if (hh == 0) reinterpret_cast<float4*>(a.part_meta)[prow] = make_float4(m, l, le, (float)ex);
    return;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint16_t* out = a.o + at * D + 4 * hh;
#pragma unroll
  for (int t = 0; t < D / 32; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<uint2*>(out + 32 * t + 8 * g) =
          make_uint2(pack2_bf16(acc[t][4 * g] * inv, acc[t][4 * g + 1] * inv),
                     pack2_bf16(acc[t][4 * g + 2] * inv, acc[t][4 * g + 3] * inv));
  if (a.lse != nullptr && hh == 0) a.lse[at] = le == 0.f ? -INFINITY : (m + log2f(le)) * 0.69314718055994530942f;
}

// ---- more than 32 query rows: one work-group per (head, range of the list, 32 NW rows),
// one wave per 32 rows, two waves per SIMD.
//
// What bounds it is the VALU: a 32x32x16 MFMA takes the time of 7.7 VALU instructions
// (two waves per SIMD), the softmax takes 4.2 of those per MFMA at D = 128, and turning
// every K and V operand into bf16 would take 4 more in each wave.  So both are turned into
// bf16 once per work-group, on the way into LDS: a wave loads its share of a raw tile into
// registers two steps ahead, converts it and stores it, K in the layout of row reads and V
// in that of the transpose read (1 conversion per MFMA and wave with four waves, 2 with
// two).  Products of codes would need no conversion of K, with Q as the sum of two e4m3
// numbers; but v_mfma_f32_32x32x64_f8f6f4 aligns the products of eight columns to the
// largest of them with 13 bits, which cost up to 8e-4 of the lse.
//
// Step t: S of tile t + 1 and P V of tile t - 1 on the matrix cores, the softmax of tile t
// spread evenly under them, K of tile t + 2 and V of tile t converted.  One barrier per
// step, P MFMAs before its end, behind which the converted tiles can be read.
// The softmax keeps a running max that is only refreshed when some lane's sum of a tile's
// P exceeds 2^8 (attn_fwd.hip); the row sum of the bf16 P comes from 4x4x4 MFMAs.  P is bf16
// because its products' other operand, V, is: the scales of neither cache fit fp16's range.  A
// weight is off by at most 2^-8 of itself and O by about as much as by its own rounding; P as
// two bf16 numbers would make 24 products of a step's 16.
//
// D = 128, N(0, 1) and random lists, ms, all on one card (the clock differs between cards by
// some 3%, and with the data: what needs fewer bits takes less power):
//                                          8 bits   4 bits   the bf16 forward
//   24 heads,  2,880 x  75,392, dense       2.66     2.60     2.56
//   24 heads, 25,920 x  98,432, dense      29.4     29.4     28.0
//   24 heads, 11,520 x  84,032, 25%         3.49     3.48     3.17
//   24 heads, 72,000 x 144,512, 25%        34.8     35.0     33.6
//   24 heads, 72,000 x 144,512, 9.4%, 128  12.6     12.9     12.7
//    8 heads, 11,520 x  84,032, 25%         1.23     1.20     1.11
//    8 heads, 11,520 x  84,032, 25%, 128    1.08     1.05     1.02
// The first is 1.02 PFLOP/s with 4 bits, the matrix cores busy half of the cycles at 1.8 GHz, the
// VALU issuing 0.10 instructions per SIMD and cycle.
template <int D, int NW>
struct CachePipe : CacheCfg<D> {
  using B = CacheCfg<D>;
  static constexpr int NA = B::KT * B::DS;      // MFMAs of S
  static constexpr int NB = 2 * B::KT * B::DT;  // MFMAs of P V
  static constexpr int NE = 16 * B::KT;         // elements of S per lane
  static constexpr int EPU = NE / 16;           // elements per MFMA
  static constexpr int CT = B::KB * D;          // elements of a converted tile
  static constexpr int CV = 4 / NW;             // 16-code pieces of a tile that a lane converts
  static constexpr int P = 4, PV = 6;           // MFMAs between a K (V) operand's read and its use
  static_assert(NA == 8 && NB == 8, "a step is 16 MFMAs");
};

// A raw buffer over `bytes` bytes, in scalar registers.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const uint8_t* p, uint32_t bytes) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)u);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((int)(uint32_t)(u >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((uint64_t)hi << 32 | lo), 0,
                                           __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}

// A barrier that makes LDS writes visible and lets LDS reads end, and waits for no load.
__device__ __forceinline__ void publish_lds() {
  __builtin_amdgcn_s_waitcnt((63 & 15) | ((63 >> 4) << 14) | (7 << 4));
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

template <int D, int NW, bool DENSE, class F>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2)))
void cache_attn_kernel(typename F::Args a) {
  using C = CachePipe<D, NW>;
  constexpr int ROWS = 32 * NW;
  __shared__ __attribute__((aligned(1024))) uint16_t kb[2][C::CT];
  __shared__ __attribute__((aligned(1024))) uint16_t vb[2][C::CT];

  // Work item: as in attn_fwd.hip, the query groups of a (head, range) pair are dealt out
  // to 2^spread_bits XCDs, each of which runs its share of a pair after the other.
  const uint32_t n_g = (uint32_t)((a.lq + ROWS - 1) / ROWS);
  uint32_t gi, pair;
  int qg;
  if (a.spread_bits == 3) {
    pair = blockIdx.x / n_g;
    qg = (int)(blockIdx.x - pair * n_g);
    gi = (uint32_t)qg >> 3;
  } else {
    const uint32_t n_u = (n_g + (1u << a.spread_bits) - 1) >> a.spread_bits;
    const uint32_t id = blockIdx.x / 8, ui = id / n_u;
    gi = id - ui * n_u;
    const uint32_t unit = ui * 8 + (blockIdx.x + ui) % 8;
    pair = unit >> a.spread_bits;
    qg = (int)((gi << a.spread_bits) + (unit & ((1u << a.spread_bits) - 1)));
  }
  if (pair >= (uint32_t)a.bh * (uint32_t)a.ranges || qg >= (int)n_g) return;  // uniform: past the last unit or group
  const int64_t bh = pair / (uint32_t)a.ranges;
  const int range = (int)(pair - (uint32_t)bh * (uint32_t)a.ranges);
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int l32 = lane % 32, hh = lane / 32;

  // tokens that exist: rows past them are neither read nor attended to
  // (both counts are loaded before either is waited for)
  int given = 0, listed = 0;
  if (a.lens != nullptr) given = a.lens[(uint32_t)bh / (uint32_t)a.heads];
  if constexpr (!DENSE) listed = a.kv_num_blocks[bh * a.n_q + qg];
  const int64_t len = a.lens == nullptr ? a.lk : (given < 0 ? 0 : (given < a.lk ? given : a.lk));
  const int block_bits = a.block == 128 ? 7 : 6;
  const int n_blk = (int)((len + a.block - 1) >> block_bits);

  // ---- Q as the B operand of S^T = K Q^T: Q[q][16 s + 8 h .. +7]
  const int64_t row = (int64_t)qg * ROWS + wave * 32 + l32;
  const bool row_ok = row < a.lq;
  bf16x8 qf[C::DS];
#pragma unroll
  for (int s = 0; s < C::DS; ++s) {
    const uint16_t* p = a.q + (bh * a.lq + (row_ok ? row : 0)) * D + 16 * s + 8 * hh;
    const uint4 u = row_ok ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0);
    qf[s] = __builtin_bit_cast(bf16x8, u);
  }

  // (dense entries are 64 keys whatever the block size)
  const int e_bits = DENSE ? (a.block == 128 ? 1 : 0) : 0;

  // ---- the range's key blocks: an even share of the list's entries, or of all blocks,
  // walked from `rot` on and around (see attn_fwd.hip for why)
  int first = 0, cnt, rot = 0;
  const int32_t* list = nullptr;
  {
    int n = n_blk;
    if constexpr (!DENSE) {
      n = listed < 0 ? 0 : (listed > a.stride ? a.stride : listed);
      list = a.kv_indices + (bh * a.n_q + qg) * a.stride;
    }
    if constexpr (DENSE && F::PAGED) n <<= e_bits;
    // (a 64-bit division is some 150 scalar instructions)
    auto part = [&](int r) -> int {
      if (n < 1 << 25) return (int)((uint32_t)n * (uint32_t)r / (uint32_t)a.ranges);
      return (int)((int64_t)n * r / a.ranges);
    };
    first = __builtin_amdgcn_readfirstlane(part(range));
    cnt = __builtin_amdgcn_readfirstlane(part(range + 1)) - first;
    if (!DENSE && a.rotation > 0 && n < n_blk)
      rot = (int)((int64_t)(gi % (uint32_t)a.rotation) * cnt / a.rotation);
  }
  // Entries 64 at a time in VGPRs: the block and its scale bytes, or its page's first tile in the
  // pool (which holds less than 2^31).  One that names no block (page) gives -1, whose tiles are
  // loaded as zeros and masked.
  constexpr int SUB = (DENSE ? 64 : ROWS) / C::KB;  // tiles per entry (dense: of 64 keys)
  const int64_t scale_at = bh * ((a.cap + a.block - 1) >> block_bits);
  int breg = -1, sreg = 0, lbase = 0;
  const int32_t* page_row = nullptr;
  int head_of = 0;
  if constexpr (F::PAGED) {
    const uint32_t seq = (uint32_t)bh / (uint32_t)a.heads;
    head_of = (int)((uint32_t)bh - seq * (uint32_t)a.heads);
    page_row = a.pages + seq * a.n_table;
  }
  if constexpr (DENSE && !F::PAGED) {  // (whole blocks, as the lists')
    first <<= e_bits;
    cnt <<= e_bits;
  }
  auto load_batch = [&](int base) {
    lbase = base;
    int b = -1;
    if (base + lane < cnt) {
      const int e = base + lane + rot;
      b = DENSE ? first + base + lane : list[first + (e >= cnt ? e - cnt : e)];
    }
    const int blk = b >> e_bits;
    if (b < 0 || blk >= n_blk) b = -1;
    if constexpr (F::PAGED) {
      const int page = b < 0 ? -1 : page_row[blk];
      if (page < 0 || page >= a.n_pages) b = -1;
      // (dense: the entry's 64 keys of the page)
      sreg = b < 0 ? 0 : (page * a.heads + head_of) * (a.block / C::KB) + (DENSE ? (b & ((1 << e_bits) - 1)) * SUB : 0);
    } else {
      sreg = 127 | 127 << 8;
      if (b >= 0) sreg = (int)a.k_scale[scale_at + blk] | (int)a.v_scale[scale_at + blk] << 8;
    }
    breg = b;
    asm volatile("; list batch %0 %1" ::"v"(breg), "v"(sreg));
  };
  const int ntiles = cnt * SUB;
  struct Tile {
    int t;  // KB-key tile of the sequence, -1: none
    int s;  // scale bytes, or the tile's place in the pool, in tiles
  };
  auto fetch = [&](int j) -> Tile {
    if (j >= ntiles) return Tile{-1, F::PAGED ? 0 : 127 | 127 << 8};
    const int e = j / SUB;
    if (e >= lbase + 64) load_batch(lbase + 64);
    const int b = __builtin_amdgcn_readlane(breg, e - lbase);
    return Tile{b < 0 ? -1 : b * SUB + j % SUB, __builtin_amdgcn_readlane(sreg, e - lbase) + (F::PAGED ? j % SUB : 0)};
  };

  // ---- raw tiles: the lane's 16-code pieces at code src + 1024 i of a tile.  Each tile gets
  // its own descriptor, so that rows past the sequence's end arrive as zeros.
  const uint32_t n_whole = (uint32_t)(len / C::KB), last_codes = (uint32_t)(len % C::KB) * D;
  const int src = 1024 * C::CV * wave + 16 * lane;
  using Piece = typename F::Piece;
  auto load_raw = [&](const uint8_t* codes, const uint8_t* scales, Tile t, Piece (&u)[C::CV]) {
    const uint32_t n = (uint32_t)t.t < n_whole ? C::KB * D : ((uint32_t)t.t == n_whole ? last_codes : 0u);
    if constexpr (F::PAGED) {
      const uint64_t at = (uint32_t)__builtin_amdgcn_readfirstlane(t.s);
      const auto rs = tile_rsrc(codes + at * (C::KB * D / 2), n / 2), rss = tile_rsrc(scales + at * (C::KB * D / 32), n / 32);
#pragma unroll
      for (int i = 0; i < C::CV; ++i) {
        u[i].u = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rs, src / 2 + 512 * i, 0, 0));
        u[i].s = __builtin_amdgcn_raw_buffer_load_b8(rss, src / 32 + 32 * i, 0, 0);
      }
    } else {
      const auto rs = tile_rsrc(codes + bh * a.cap * D + (int64_t)t.t * C::TILE, n);
#pragma unroll
      for (int i = 0; i < C::CV; ++i)
        u[i].u = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(rs, src + 1024 * i, 0, 0));
    }
  };
  auto load_k = [&](Tile t, Piece (&u)[C::CV]) { load_raw(a.k_cache, a.k_scale, t, u); };
  auto load_v = [&](Tile t, Piece (&u)[C::CV]) { load_raw(a.v_cache, a.v_scale, t, u); };

  // ---- converted tiles: rows of 2 D bytes whose 16-byte chunks are permuted as in
  // attn_fwd.hip, chunk c of K row r at c ^ kswz(r), of V row r at c ^ vswz(r).  A store of 16
  // bytes a lane takes eight lanes at a time, over 128 bytes of banks: a lane's first piece is
  // an even chunk, so those of the second half of 256 bytes are moved to the odd ones (without
  // it every store took twice its eight cycles, an eighth of the dense kernel's cycles).
  constexpr int CRB = 2 * D, CRPB = 256 / CRB, CCPR = D / 8;
  auto kswz = [](int r) { return (r / CRPB) % CCPR; };
  auto vswz = [](int r) { return (((r / CRPB) & 3) << 2) & (CCPR - 1); };
  auto half = [](int r, int c) { return D == 128 ? c >> 3 : r & 1; };
  uint32_t koff[C::DS];  // K row l32, chunk 2 s + h
#pragma unroll
  for (int s = 0; s < C::DS; ++s) koff[s] = (uint32_t)(l32 * CRB + 16 * ((2 * s + hh) ^ kswz(l32) ^ half(l32, 2 * s + hh)));
  uint32_t voff[C::DT];  // transpose read: rows 4 h + (0..3), columns 32 t + l % 32
  {
    const int sl = lane & 15, r = 4 * hh + (sl >> 2);
#pragma unroll
    for (int t = 0; t < C::DT; ++t) {
      const int c = 4 * t + 2 * (lane >> 4 & 1) + ((sl & 3) >> 1);
      voff[t] = (uint32_t)(r * CRB + 16 * (c ^ vswz(r) ^ half(r, c)) + 8 * (sl & 1));
    }
  }
  // Where the lane's pieces go: to two neighbouring chunks, 8 (D = 64: 16) rows further per
  // i, which moves kswz by 8 chunks of 16 (D = 128) or not at all, and leaves vswz as it is.
  uint32_t kdst, vdst;
  {
    const int r = src / D, c = 2 * (src % D / 16);
    kdst = (uint32_t)(r * CRB + 16 * (c ^ kswz(r) ^ half(r, c)));
    vdst = (uint32_t)(r * CRB + 16 * (c ^ vswz(r) ^ half(r, c)));
  }
  auto convert = [&](const Piece& p, int byte, char* tile, uint32_t dst) {
    if constexpr (F::PAGED) {
      const float sc = __uint_as_float(p.s << 23);
      *reinterpret_cast<bf16x8*>(tile + dst) = decode8_4bit(p.u.x, sc);
      *reinterpret_cast<bf16x8*>(tile + (dst ^ 16u)) = decode8_4bit(p.u.y, sc);
    } else {
      const float sc = __uint_as_float((uint32_t)(byte & 255) << 23);
      *reinterpret_cast<bf16x8*>(tile + dst) = decode8(make_uint2(p.u.x, p.u.y), sc);
      *reinterpret_cast<bf16x8*>(tile + (dst ^ 16u)) = decode8(make_uint2(p.u.z, p.u.w), sc);
    }
  };
  auto convert_k = [&](const Piece& u, int i, int s, int buf) {
    convert(u, s, reinterpret_cast<char*>(kb[buf]) + 2048 * i, D == 128 ? kdst ^ (uint32_t)(128 * (i % 2)) : kdst);
  };
  auto convert_v = [&](const Piece& u, int i, int s, int buf) {
    convert(u, s >> 8, reinterpret_cast<char*>(vb[buf]) + 2048 * i, vdst);
  };

  const s16x4 one4 = {0x3f80, 0x3f80, 0x3f80, 0x3f80};  // bf16 1.0
  auto mask_tile = [&](f32x16* x, int tile) {
    const int64_t left = tile < 0 ? 0 : len - (int64_t)tile * C::KB;
    const int vis = (int)(left < 0 ? 0 : (left > C::KB ? C::KB : left)) - 4 * hh;
    asm volatile("; mask");  // (keeps the branch around this: it is rarely taken)
#pragma unroll
    for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (kt * 32 + 8 * (e / 4) + (e % 4) >= vis) x[kt][e] = -INFINITY;
  };
  auto tile_max = [&](const f32x16* x) -> float {
    float mx = -INFINITY;
#pragma unroll
    for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, x[kt][e]);
    return mx;
  };
  const float sl2 = a.scale_log2;

  f32x16 acc[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f, le_run = 0.f;  // max in the log2 domain; sums of the lane's half of the keys

  if (ntiles > 0) {
    // K operand of MFMA n = kt DS + s of S
    auto read_k = [&](int n, int buf) -> bf16x8 {
      return __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(kb[buf]) +
                                                                        koff[n % C::DS] + n / C::DS * 32 * CRB));
    };
    // V^T operand of P V: step m = (2 kt + half) DT + dt
    auto read_v = [&](int m, int buf) -> bf16x8 {
      typedef __attribute__((address_space(3))) uint16_t lds16;
      const lds16* p = (const lds16*)vb[0] + (voff[m % C::DT] / 2 + 16 * (m / C::DT) * D + buf * C::CT);
      const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
      const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p + 8 * D));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // ---- prologue: K of tiles 0 and 1 converted, S of tile 0, raw tiles in flight
    load_batch(0);
    Tile t0 = fetch(0), t1 = fetch(1), t2 = fetch(2), t3 = fetch(3);
    Piece kraw[2][C::CV], vraw[2][C::CV];  // of tiles t + 2 and t + 3, t and t + 1
    load_k(t0, kraw[0]);
    load_k(t1, kraw[1]);
    load_v(t0, vraw[0]);
    load_v(t1, vraw[1]);
#pragma unroll
    for (int i = 0; i < C::CV; ++i) {
      convert_k(kraw[0][i], i, t0.s, 0);
      convert_k(kraw[1][i], i, t1.s, 1);
    }
    load_k(t2, kraw[0]);
    load_k(t3, kraw[1]);
    // "P V of tile -1" multiplies zeros
    for (int i = threadIdx.x; i < C::CT / 8; i += 64 * NW) reinterpret_cast<uint4*>(vb[1])[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    f32x16 s[C::KT];  // S^T of tile t
#pragma unroll
    for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
      for (int e = 0; e < 16; ++e) s[kt][e] = 0.f;
    static_for<C::NA>([&](auto nc) {
      constexpr int n = decltype(nc)::value, kt = n / C::DS;
      s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_k(n, 0), qf[n % C::DS], s[kt], 0, 0, 0);
    });
    if ((uint32_t)t0.t >= n_whole) mask_tile(s, t0.t);
    m_run = half_swap_max(tile_max(s)) * sl2;  // O and the sums are still zero
    u32x8 pp[C::KT];                           // bf16 pairs of P^T of tile t - 1
#pragma unroll
    for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
      for (int i = 0; i < 8; ++i) pp[kt][i] = 0u;
    bf16x8 ahead[C::P];                        // K operands of the next MFMAs
#pragma unroll
    for (int i = 0; i < C::P; ++i) ahead[i] = read_k(i, 1);
    __syncthreads();  // the first step overwrites K of tile 0

    int j = 0;
    auto step = [&](auto tc) {
      // t mod 2: the buffer of K(t), which K(t + 2) takes, and of V(t)
      constexpr int T = decltype(tc)::value, U = 1 - T;
      constexpr int X = C::NA + C::NB - C::P;  // MFMA before which the barrier stands
      f32x16 sn[C::KT];
      u32x8 pk[C::KT];
      bf16x8 kop[C::NA + C::P], vop[C::NB];
      float x[C::NE], p[C::NE], se = 0.f;
      f32x4 st4 = {0.f, 0.f, 0.f, 0.f};
      const float neg_m = m_run == -INFINITY ? INFINITY : -m_run;  // (no key seen yet: takes the exact path)
#pragma unroll
      for (int i = 0; i < C::P; ++i) kop[i] = ahead[i];
      auto row_sum = [&](auto ic) {  // adds pairs i - 1 and i of P
        constexpr int i = decltype(ic)::value;
        const uint2 u = make_uint2(pk[i / 8][i % 8 - 1], pk[i / 8][i % 8]);
        st4 = __builtin_amdgcn_mfma_f32_4x4x4bf16_1k(one4, __builtin_bit_cast(s16x4, u), st4, 0, 0, 0);
      };
      auto logit = [&](auto ec) {
        constexpr int e = decltype(ec)::value;
        if constexpr (e < C::NE) {
          x[e] = fmaf(s[e / 16][e % 16], sl2, neg_m);
          asm volatile("" : "+v"(x[e]));  // holds the work here (it would otherwise sink to its uses)
        }
      };
      auto prob = [&](auto ec) {
        constexpr int e = decltype(ec)::value;
        if constexpr (e < C::NE) {
          p[e] = __builtin_amdgcn_exp2f(x[e]);
          asm volatile("" : "+v"(p[e]));
        }
      };
      auto element = [&](auto ec) {  // each stage works one element behind the stage before
        constexpr int e = decltype(ec)::value;
        logit(std::integral_constant<int, e + 2>{});
        prob(std::integral_constant<int, e + 1>{});
        se = e == 0 ? p[0] : se + p[e];
        asm volatile("" : "+v"(se));
        if constexpr (e % 2 == 1) pk[e / 16][e % 16 / 2] = pack2_bf16(p[e - 1], p[e]);
      };
      logit(std::integral_constant<int, 0>{});
      logit(std::integral_constant<int, 1>{});
      prob(std::integral_constant<int, 0>{});
      __builtin_amdgcn_sched_barrier(0);
      static_for<C::NA + C::NB>([&](auto nc) {
        constexpr int n = decltype(nc)::value;
        if constexpr (n < C::NA) {  // S of tile t + 1
          constexpr int kt = n / C::DS;
          if constexpr (n % C::DS == 0)
#pragma unroll
            for (int e = 0; e < 16; ++e) sn[kt][e] = 0.f;
          sn[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kop[n], qf[n % C::DS], sn[kt], 0, 0, 0);
        } else {  // P V of tile t - 1
          constexpr int m = n - C::NA, kt = m / C::DT / 2, half = m / C::DT % 2, dt = m % C::DT;
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vop[m], pack_half(pp[kt], half), acc[dt], 0, 0, 0);
        }
        // the converted tiles can be read behind the barrier, those of the step before
        // overwritten
        if constexpr (n == X - 1) publish_lds();
        constexpr int rk = n + C::P, rv = n + C::PV - C::NA;
        if constexpr (rk < C::NA) kop[rk] = read_k(rk, U);
        if constexpr (rk >= C::NA + C::NB) kop[rk - C::NB] = read_k(rk - C::NA - C::NB, T);
        if constexpr (rv >= 0 && rv < C::NB) vop[rv] = read_v(rv, U);
        // K of tile t + 2 and V of tile t, a piece at a time; their registers take the raw
        // pieces of two tiles on
        if constexpr (n % 2 == 0 && n / 2 < C::CV) convert_k(kraw[T][n / 2], n / 2, t2.s, T);
        if constexpr (n % 2 == 0 && n >= 4 && n / 2 - 2 < C::CV) convert_v(vraw[T][n / 2 - 2], n / 2 - 2, t0.s, T);
        static_for<C::EPU>([&](auto k) { element(std::integral_constant<int, n * C::EPU + decltype(k)::value>{}); });
        __builtin_amdgcn_sched_barrier(0);
      });
      static_for<C::NE / 4>([&](auto k) { row_sum(std::integral_constant<int, 2 * decltype(k)::value + 1>{}); });
      float st = st4[0];
      const Tile t4 = fetch(j + 4);
      load_v(t2, vraw[T]);
      load_k(t4, kraw[T]);

      // A lane's sum of its P stays <= 2^8 whenever every p does; otherwise the exact path:
      // the tile's max, a rescale of O (tiles up to t - 1) and both sums, and P again.
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(st <= 256.f)) != 0, 0)) {
        const float mx = half_swap_max(tile_max(s)) * sl2;
        if (mx > m_run) {
          float alpha = 0.f;
          const float dm = mx - m_run;
          if (dm > 128.f) {
            m_run = mx;
          } else {
            const float k = ceilf(dm);
            alpha = __builtin_amdgcn_ldexpf(1.f, -(int)k);
            m_run += k;
          }
          l_run *= alpha;
          le_run *= alpha;
#pragma unroll
          for (int d = 0; d < C::DT; ++d)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[d][e] *= alpha;
        }
        st = 0.f;
        se = 0.f;
        const float off = m_run == -INFINITY ? 0.f : -m_run;
#pragma unroll
        for (int e = 0; e < C::NE; e += 2) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[e / 16][e % 16], sl2, off));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(s[e / 16][e % 16 + 1], sl2, off));
          se += p0;
          se += p1;
          const uint32_t u = pack2_bf16(p0, p1);
          st += bf16_lo(u) + bf16_hi(u);
          pk[e / 16][e % 16 / 2] = u;
        }
      }
      l_run += st;
      le_run += se;
      if (__builtin_expect((uint32_t)t1.t >= n_whole, 0)) mask_tile(sn, t1.t);
#pragma unroll
      for (int kt = 0; kt < C::KT; ++kt) {
        s[kt] = sn[kt];
        pp[kt] = pk[kt];
      }
#pragma unroll
      for (int i = 0; i < C::P; ++i) ahead[i] = kop[C::NA + i];
      t0 = t1;
      t1 = t2;
      t2 = t3;
      t3 = t4;
    };
    while (true) {
      step(std::integral_constant<int, 0>{});
      if (++j >= ntiles) break;
      step(std::integral_constant<int, 1>{});
      if (++j >= ntiles) break;
    }
    // P V of the last tile, which the last step converted and published
#pragma unroll
    for (int m = 0; m < C::NB; ++m)
      acc[m % C::DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
          read_v(m, (ntiles - 1) % 2), pack_half(pp[m / C::DT / 2], m / C::DT % 2), acc[m % C::DT], 0, 0, 0);
  }
  store_rows<D, F>(a, bh, row, range, acc, m_run, half_swap_sum(l_run), half_swap_sum(le_run), hh);
}

// Joins the ranges of one row: with M = max_r m_r and w_r = 2^(m_r - M),
// O = sum w_r 2^e_r A_r / sum w_r l_r and lse = ln 2 (M + log2 sum w_r le_r).  D / 8 threads
// per row and G groups of them, each over every G-th range; the groups' own sums are joined
// the same way through LDS.  Groups suit many ranges of few rows, one group many rows (64 rows
// in 64 ranges 4.0 us with 16 groups, 16.5 with one; 14,400 in 8 19 and 7.4).
template <int D, int G, class F>
__global__ __launch_bounds__(256) void cache_merge_kernel(typename F::Args a) {
  constexpr int LPR = D / 8, RPB = 256 / (LPR * G);
  __shared__ float red[G][RPB][LPR][8], meta[G][RPB][3];
  const int c = threadIdx.x % LPR, g = threadIdx.x / LPR % G, rb = threadIdx.x / (LPR * G);
  const int64_t rows = (int64_t)a.bh * a.lq, row = (int64_t)blockIdx.x * RPB + rb;
  const bool ok = row < rows;
  float m = -INFINITY, l = 0.f, le = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (ok) {
    // (four ranges' loads at once: with one after the other their latency was half of the time)
    for (int r0 = 0; r0 < a.ranges; r0 += 4 * G) {
      float4 x[4];
      typename F::Part u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = make_float4(0.f, 0.f, 0.f, 0.f), u[i] = typename F::Part{0, 0, 0, 0, 0, 0, 0, 0};
        if (r0 + i * G >= a.ranges) continue;
        const int64_t p = (int64_t)min(r0 + i * G + g, a.ranges - 1) * rows + row;
        x[i] = reinterpret_cast<const float4*>(a.part_meta)[p];
        u[i] = reinterpret_cast<const typename F::Part*>(a.part_o)[p * LPR + c];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (r0 + i * G + g >= a.ranges || x[i].y == 0.f) continue;  // no key seen; NaN passes on
        const float mn = fmaxf(m, x[i].x), s = __builtin_amdgcn_exp2f(m - mn), t = __builtin_amdgcn_exp2f(x[i].x - mn);
        const float w = __builtin_amdgcn_ldexpf(t, (int)x[i].w);
        l = l * s + x[i].y * t;
        le = le * s + x[i].z * t;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = fmaf(w, (float)u[i][e], acc[e] * s);
        m = mn;
      }
    }
  }
  if constexpr (G > 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) red[g][rb][c][e] = acc[e];
    if (c == 0) meta[g][rb][0] = m, meta[g][rb][1] = l, meta[g][rb][2] = le;
    __syncthreads();
    if (g != 0) return;
    float mm = m;
#pragma unroll
    for (int i = 1; i < G; ++i) mm = fmaxf(mm, meta[i][rb][0]);
    // (a group without keys has m = -inf, and so has mm if none has any)
    auto weight = [&](float x) { return x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x - mm); };
    float s = weight(m);
    l = l == 0.f ? 0.f : l * s, le = le == 0.f ? 0.f : le * s;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] = acc[e] * s;
#pragma unroll
    for (int i = 1; i < G; ++i) {
      s = weight(meta[i][rb][0]);
      l = fmaf(meta[i][rb][1], s, l);
      le = fmaf(meta[i][rb][2], s, le);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = fmaf(red[i][rb][c][e], s, acc[e]);
    }
    m = mm;
  }
  if (!ok) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<uint4*>(a.o + row * D + 8 * c) =
      make_uint4(pack2_bf16(acc[0] * inv, acc[1] * inv), pack2_bf16(acc[2] * inv, acc[3] * inv),
                 pack2_bf16(acc[4] * inv, acc[5] * inv), pack2_bf16(acc[6] * inv, acc[7] * inv));
  if (a.lse != nullptr && c == 0) a.lse[row] = le == 0.f ? -INFINITY : (m + log2f(le)) * 0.69314718055994530942f;
}

template <int D, int G, class F>
static hipError_t launch_merge(const typename F::Args& a, hipStream_t stream) {
  constexpr int RPB = 256 / (D / 8 * G);
  const int64_t rows = (int64_t)a.bh * a.lq;
  if (a.ranges > 1) cache_merge_kernel<D, G, F><<<(rows + RPB - 1) / RPB, 256, 0, stream>>>(a);
  return hipGetLastError();
}

// The launches of a call of more than 32 rows.
template <int D, bool DENSE, class F>
static hipError_t launch_rows(const typename F::Args& a, int waves, int join_groups, hipStream_t stream) {
  if (waves == 2) cache_attn_kernel<D, 2, DENSE, F><<<a.grid, 128, 0, stream>>>(a);
  else cache_attn_kernel<D, 4, DENSE, F><<<a.grid, 256, 0, stream>>>(a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if constexpr (F::PAGED) {
    if (join_groups == 4) return launch_merge<D, 4, F>(a, stream);
  }
  return join_groups > 1 ? launch_merge<D, 16, F>(a, stream) : launch_merge<D, 1, F>(a, stream);
}

}  // namespace sparstar
