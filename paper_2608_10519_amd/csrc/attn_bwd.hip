// Gradients of the block-sparse and the dense attention forward.
//
// With P_tu = exp(s q_t . k_u - lse_t) over the keys u that query t attends to,
//   delta_t = sum_d dO_td O_td - dlse_t
//   dP_tu   = dO_t . v_u             dS_tu = P_tu (dP_tu - delta_t)
//   dV_u    = sum_t P_tu dO_t        dK_u  = s sum_t dS_tu q_t
//   dQ_t    = s sum_u dS_tu k_u
// P is recomputed from the lse that the forward left, so nothing of size Lq x Lk
// is ever stored.
//
// Two passes, each of which owns what it writes: one work-group per query group
// walks its keys and sums dQ (three products per tile), one per key group walks
// the query blocks that list it and sums dK and dV (four products).  The five
// products of a single pass would need dQ summed over work-groups by atomics, in
// an order that changes from call to call, and its traffic, 32 KB per 64 x 64
// tile, is several times what the matrix cores take for the tile.  The results
// here are the same bits every time.
//
// The key groups find their query blocks in a bit matrix, one bit per (key block,
// query block), that a small kernel builds from the lists.
//
// What bounds it: the matrix products, 14 D operations per pair of query and key where 10
// would do in one pass, at the clock that the chip holds under them (1.55 GHz in the dense
// dQ pass, its matrix cores busy 77% of the cycles; 1.81 GHz and 61% in dK/dV; a large
// library product 1.85 and 70%).  24 dense heads of 2,880 x 75,392: 7.64 ms, 1.22 PFLOP/s
// executed, of 1.29 that a large product reaches; 3 heads of 72,000 x 144,512 at 9.4%, block
// 128: 4.8 ms, 1.14 PFLOP/s; at D = 64, where an element's softmax serves half the products,
// 1.08 (24 dense heads of 2,880 x 75,392, 4.32 ms, matrix cores 57% and 62% busy) and 0.92 (2 x
// 3 heads of 11,001 x 31,818, 1.01 ms: lists of different lengths leave CUs idle 14% and 24%).
#include "attn_device.h"

namespace sparstar {

// Tiles of 32 rows.  Rows are stored unpadded in LDS and their 16-byte chunks XOR-permuted
// by swz(row), which leaves both reads of a tile free of bank conflicts: 16 consecutive rows
// of one chunk (ds_read_b128), and four consecutive rows of four chunks (the transpose read).
template <int D>
struct BwdCfg {
  static constexpr int KB = 32;                 // rows per tile
  static constexpr int DS = D / 16;             // MFMA k-steps over D
  static constexpr int DT = D / 32;             // 32-row tiles of a D-row result
  static constexpr int RB = D * 2;              // bytes per row
  static constexpr int CPR = D / 8;             // 16-byte chunks per row
  static constexpr int RPD = 1024 / RB;         // rows per direct-to-LDS wave load
  static constexpr int TILE = KB * D;           // elements per tile
  static constexpr int TILE_BYTES = TILE * 2;
};

template <int D>
__device__ __forceinline__ int bwd_swz(int r) {
  return D == 128 ? ((r & 3) << 2 | ((r >> 2) & 3)) : (((r >> 1) & 1) << 2 | ((r >> 2) & 3));
}

// Per-lane LDS byte offsets within a tile (see attn_fwd.hip for the layouts):
// row[s]: row l % 32, the k-step's 8 columns (A operand of a product over D);
// tr[i][t]: the transpose read of rows 4 h + 8 i + (0..3), columns 32 t + l % 32.
template <int D>
struct BwdOffsets {
  using C = BwdCfg<D>;
  uint32_t row[C::DS];
  uint32_t tr[2][C::DT];
  __device__ __forceinline__ explicit BwdOffsets(int lane) {
    const int l32 = lane % 32, hh = lane / 32, grp = lane >> 4, sl = lane & 15;
#pragma unroll
    for (int s = 0; s < C::DS; ++s) row[s] = (uint32_t)(l32 * C::RB + 16 * ((2 * s + hh) ^ bwd_swz<D>(l32)));
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int t = 0; t < C::DT; ++t) {
        const int r = 4 * hh + 8 * i + (sl >> 2);
        const int c = 4 * t + 2 * (grp & 1) + ((sl & 3) >> 1);
        tr[i][t] = (uint32_t)(r * C::RB + 16 * (c ^ bwd_swz<D>(r)) + 8 * (sl & 1));
      }
  }
};

__device__ __forceinline__ const uint16_t* lds_at(const uint16_t* tile, uint32_t bytes) {
  return reinterpret_cast<const uint16_t*>(reinterpret_cast<const char*>(tile) + bytes);
}

template <int D>
__device__ __forceinline__ bf16x8 tile_row(const uint16_t* tile, const BwdOffsets<D>& off, int kt, int s) {
  return __builtin_bit_cast(
      bf16x8, *reinterpret_cast<const uint4*>(lds_at(tile, off.row[s] + kt * 32 * BwdCfg<D>::RB)));
}

// rows 32 kt + 16 half + (4 h + 0..3, 8 + 4 h + 0..3), columns 32 t + l % 32
template <int D>
__device__ __forceinline__ bf16x8 tile_col(const uint16_t* tile, const BwdOffsets<D>& off, int kt, int half, int t) {
  const uint32_t base = (uint32_t)((32 * kt + 16 * half) * BwdCfg<D>::RB);
  const s16x4 v0 = lds_read_tr(lds_at(tile, off.tr[0][t] + base));
  const s16x4 v1 = lds_read_tr(lds_at(tile, off.tr[1][t] + base));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ bf16x8 load_row(const uint16_t* p, bool ok) {
  const uint4 u = ok ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0);
  return __builtin_bit_cast(bf16x8, u);
}

// Which rows of a [rows, D] tensor a tile holds: tiles below `whole` lie inside it, tile
// `whole` holds what is left, and later ones (and -1) hold nothing.
template <class C>
struct TileRows {
  uint32_t whole, last_bytes;
  __device__ __forceinline__ explicit TileRows(int64_t rows)
      : whole((uint32_t)(rows / C::KB)), last_bytes((uint32_t)(rows % C::KB) * (uint32_t)C::RB) {}
  __device__ __forceinline__ uint32_t bytes(int tile) const {
    return (uint32_t)tile < whole ? (uint32_t)C::TILE_BYTES : ((uint32_t)tile == whole ? last_bytes : 0u);
  }
};

// The direct-to-LDS loads of one tile by NW waves; rows that do not exist arrive as zeros.
template <class C, int NW>
struct TileLoad {
  static constexpr int D = C::RB / 2;
  static constexpr int N = C::TILE_BYTES / 1024 / NW;  // 1 KB loads per wave
  uint32_t off[N];
  __device__ __forceinline__ TileLoad(int wave, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = C::RPD * (N * wave + i) + lane / C::CPR;
      // (the instruction adds 1024 i)
      off[i] = (uint32_t)(r * C::RB + 16 * ((lane % C::CPR) ^ bwd_swz<D>(r)) - 1024 * i);
    }
  }
  // the tile's descriptor, and its loads
  __device__ __forceinline__ static i32x4 rsrc(const uint16_t* base, int tile, uint32_t bytes) {
    return raw_rsrc(base + (int64_t)tile * C::TILE, bytes);
  }
  __device__ __forceinline__ void issue(i32x4 rs, uint16_t* slot, int wave) const {
    dma_tile<N>(lds_addr(slot) + (uint32_t)(N * wave) * 1024u, off, rs);
  }
};

// 64 consecutive floats into LDS (lane l: 4 bytes at +4 l)
__device__ __forceinline__ void dma_floats(i32x4 rs, float* slot, int lane) {
  const uint32_t voff = (uint32_t)lane * 4u;
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "buffer_load_dword %1, %2, 0 offen lds"
      :
      : "s"(lds_addr(slot)), "v"(voff), "s"(rs)
      : "memory", "m0");
}

// The barrier of a step: the tile that the wave waits for has landed and can be read by
// all, and every wave is done with the tile that the loads after it overwrite.  (Its reads
// were consumed by MFMAs long before: no wait for LDS is needed.)
__device__ __forceinline__ void publish() {
  wait_vmcnt<0>();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---- per-row statistics.  Rows are kept in groups of 32, [32] of -lse / s (what an
// unscaled logit is offset by) then [32] of -delta, padded to whole query blocks: a row past Lq,
// and one that saw no key, gets -inf and 0, which makes its P and dS zero.
template <int D>
__device__ __forceinline__ void row_stats(const BwdArgs& a, int64_t group) {
  constexpr int LPR = D / 8, RPW = 256 / LPR;
  const int64_t rows_pad = (int64_t)a.n_q * a.block;
  const int64_t i = group * RPW + threadIdx.x / LPR;
  if (i >= a.bh * rows_pad) return;
  const int64_t bh = i / rows_pad, t = i - bh * rows_pad;
  const int c = threadIdx.x % LPR;
  float sum = 0.f;
  const bool in = t < a.lq;
  const int64_t r = bh * a.lq + t;
  if (in) {
    const uint4 x = *reinterpret_cast<const uint4*>(a.o + r * D + 8 * c);
    const uint4 y = *reinterpret_cast<const uint4*>(a.d_o + r * D + 8 * c);
    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sum = fmaf(bf16_lo(xs[e]), bf16_lo(ys[e]), sum);
      sum = fmaf(bf16_hi(xs[e]), bf16_hi(ys[e]), sum);
    }
  }
#pragma unroll
  for (int w = LPR / 2; w > 0; w /= 2) sum += __shfl_xor(sum, w, LPR);
  if (c == 0) {
    float nl = -INFINITY, nd = 0.f;
    if (in) {
      const float l = a.lse[r];
      if (l != -INFINITY) {
        nl = -l * a.inv_scale;
        nd = (a.dlse != nullptr ? a.dlse[r] : 0.f) - sum;
      }
    }
    float* st = a.stats + (i / 32) * 64 + i % 32;
    st[0] = nl;
    st[32] = nd;
  }
}

// ---- the bit matrix: word w of key block j holds, bit i, whether query block
// 32 w + i lists j.  One work-group per word column and up to kBitsChunk key blocks.
__device__ __forceinline__ void list_bits(const BwdArgs& a, int64_t column, int chunk, uint32_t* bits) {
  const int64_t bh = column / a.n_words;
  const int word = (int)(column - bh * a.n_words);
  const int lo = chunk * kBitsChunk;
  const int hi = a.n_k - lo < kBitsChunk ? a.n_k : lo + kBitsChunk;
  for (int j = threadIdx.x; j < hi - lo; j += 256) bits[j] = 0u;
  __syncthreads();
  const int lane = threadIdx.x % 64;
  for (int i = threadIdx.x / 64; i < 32; i += 4) {
    const int qb = 32 * word + i;
    if (qb >= a.n_q) break;
    const int64_t r = bh * a.n_q + qb;
    int n = a.kv_num_blocks[r];
    n = n < 0 ? 0 : (n > a.stride ? a.stride : n);
#pragma unroll 4
    for (int e = lane; e < n; e += 64) {
      const int j = a.kv_indices[r * a.stride + e];
      if (j >= lo && j < hi) atomicOr(&bits[j - lo], 1u << i);
    }
  }
  __syncthreads();
  for (int j = threadIdx.x; j < hi - lo; j += 256) a.bits[(bh * a.n_k + lo + j) * a.n_words + word] = bits[j];
}

// ---- the key blocks that are taken first: 8 threads per block count its bits and cut it
// where the rank of a bit, not its place, is a multiple of count / pieces: query blocks that
// list a key block are often neighbours, and an even share of all query blocks would leave
// one piece with most of the work.  Where a block's pieces stand in the list differs from
// call to call, what is computed for them does not.
__global__ __launch_bounds__(256) void attn_bwd_pieces_kernel(BwdArgs a) {
  const int64_t n = (int64_t)a.bh * a.n_k, i = (int64_t)blockIdx.x * 32 + threadIdx.x / 8;
  const int t = threadIdx.x % 8;
  const uint32_t* const words = a.bits + i * a.n_words;
  int count = 0;
  if (i < n)
    for (int w = t; w < a.n_words; w += 8) count += __builtin_popcount(words[w]);
#pragma unroll
  for (int s = 4; s > 0; s /= 2) count += __shfl_xor(count, s, 8);
  if (i >= n) return;
  if (t == 0) a.listed[i] = count > a.list_min;
  if (count <= a.list_min) return;
  const int pieces = (count + a.piece_max - 1) / a.piece_max;
  int at = 0, slot = 0;
  if (t == 0) {
    at = atomicAdd(a.piece_count, pieces);
    if (pieces > 1) slot = atomicAdd(a.piece_count + 1, pieces);
  }
  BwdPiece* const out = a.pieces + __shfl(at, 0, 8);
  slot = __shfl(slot, 0, 8);
  for (int p = t; p < pieces; p += 8) {
    out[p].block = (int)i;
    out[p].piece = p;
    out[p].pieces = pieces;
    out[p].slot = slot + p;
  }
  if (t == 0) {
    out[0].begin = 0;
    out[pieces - 1].end = a.n_q;
  }
  if (pieces == 1) return;
  int before = 0;  // bits of the words before
  for (int w0 = 0; w0 < a.n_words; w0 += 8) {
    uint32_t left = w0 + t < a.n_words ? words[w0 + t] : 0u;
    const int c = __builtin_popcount(left);
    int upto = c;
#pragma unroll
    for (int s = 1; s < 8; s *= 2) {
      const int x = __shfl_up(upto, s, 8);
      if (t >= s) upto += x;
    }
    // pieces (but the first) that begin in this word, with the bit of rank count p / pieces
    int rank = before + upto - c;
    const int end = rank + c;
    for (int64_t p = std::max<int64_t>(1, ((int64_t)rank * pieces + count - 1) / count); p < pieces; ++p) {
      const int r = (int)((int64_t)count * p / pieces);
      if (r >= end) break;
      for (; rank < r; ++rank) left &= left - 1;
      out[p].begin = out[p - 1].end = 32 * (w0 + t) + __builtin_ctz(left);
    }
    before += __shfl(upto, 7, 8);
  }
}

// Statistics and bits in one launch: the first `stat_groups` work-groups take the rows.
template <int D>
__global__ __launch_bounds__(256) void attn_bwd_prepare_kernel(BwdArgs a, int64_t stat_groups, int chunks) {
  __shared__ uint32_t bits[kBitsChunk];
  if (a.list_min > 0 && blockIdx.x == 0 && threadIdx.x < 2) a.piece_count[threadIdx.x] = 0;
  if (blockIdx.x < stat_groups) {
    row_stats<D>(a, blockIdx.x);
  } else {
    const int64_t i = blockIdx.x - stat_groups, column = i / chunks;
    list_bits(a, column, (int)(i - column * chunks), bits);
  }
}

// Order of the work.  The dense passes give each XCD (and its L2) whole heads.  The sparse
// ones go through a head on all XCDs at once, because the heads' lists differ in length:
// with budgets from 0.5 to 1.5 of the mean, 24 heads, 11,520 queries, 84,032 keys, an XCD
// per three heads took 14.0 ms, all XCDs per head 11.2 (equal budgets: 10.1 and 10.3).

// ---- dQ: one work-group per (head, list range, query group of 32 NW rows), one
// wave per 32 rows.  Per 32-key tile S^T = K Q^T and dP^T = V dO^T (lane: 16 keys of
// one query), then dQ^T += K^T dS^T with dS rounded to bf16 once.  The step is that of
// the dK/dV pass below: S and dP of tile t + 1, then dQ of tile t, 24 MFMAs at D = 128.
template <int D>
struct DqCfg : BwdCfg<D> {
  using B = BwdCfg<D>;
  static constexpr int NA = 2 * B::DS, NB = 2 * B::DT, NM = NA + NB;  // MFMAs of a step
  static constexpr int SPREAD = NA + B::DT - 1;    // MFMAs that the softmax is spread over
  static constexpr int P = 4;                      // MFMAs between an operand's read and its use
  static constexpr int RING = 4;                   // tiles in LDS, K and V each
  // dP starts from -delta, held in 16 registers, where there are as many; else it is
  // added per element
  static constexpr bool START = D == 64;
};

template <int D>
struct alignas(1024) DqLds {
  uint16_t ks[DqCfg<D>::RING][DqCfg<D>::TILE], vs[DqCfg<D>::RING][DqCfg<D>::TILE];
};

// (index: of groups work-groups)
template <int D, int NW, bool DENSE>
__device__ __forceinline__ void attn_bwd_dq(const BwdArgs& a, DqLds<D>& lds, uint32_t index, uint32_t groups) {
  using C = DqCfg<D>;
  constexpr int ROWS = 32 * NW, SUB = ROWS / C::KB;  // (sparse: a list entry is SUB tiles)
  auto& ks = lds.ks;
  auto& vs = lds.vs;
  const int64_t n_g = (a.lq + ROWS - 1) / ROWS;
  const int64_t w = DENSE ? xcd_linear(index, groups) : index;
  const int64_t pair = w / n_g;
  const int qg = (int)(w - pair * n_g);
  const int64_t bh = pair / a.dq_ranges;
  const int range = (int)(pair - bh * a.dq_ranges);
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int l32 = lane % 32, hh = lane / 32;

  const int64_t row = (int64_t)qg * ROWS + wave * 32 + l32;
  const bool row_ok = row < a.lq;
  bf16x8 qf[C::DS], dof[C::DS];
  {
    const int64_t at = (bh * a.lq + (row_ok ? row : 0)) * D + 8 * hh;
#pragma unroll
    for (int s = 0; s < C::DS; ++s) {
      qf[s] = load_row(a.q + at + 16 * s, row_ok);
      dof[s] = load_row(a.d_o + at + 16 * s, row_ok);
    }
  }
  float nl = -INFINITY;
  float nd = 0.f;
  {
    if (row_ok) {
      const int64_t i = bh * a.n_q * a.block + row;
      nl = a.stats[(i / 32) * 64 + i % 32] * a.scale_log2;
      nd = a.stats[(i / 32) * 64 + 32 + i % 32];
    }
  }
  f32x16 start;  // where each dP of the lane's query starts from
#pragma unroll
  for (int e = 0; e < 16; ++e) start[e] = C::START ? nd : 0.f;

  // the range's entries of the list (or key tiles of the dense call)
  int first = 0, cnt;
  const int32_t* list = nullptr;
  if constexpr (DENSE) {
    const int64_t n = (a.lk + C::KB - 1) / C::KB;
    first = (int)(n * range / a.dq_ranges);
    cnt = (int)(n * (range + 1) / a.dq_ranges) - first;
  } else {
    const int64_t r = bh * a.n_q + qg;
    int n = a.kv_num_blocks[r];
    n = n < 0 ? 0 : (n > a.stride ? a.stride : n);
    const int p0 = (int)((int64_t)n * range / a.dq_ranges);
    cnt = (int)((int64_t)n * (range + 1) / a.dq_ranges) - p0;
    cnt = __builtin_amdgcn_readfirstlane(cnt);
    list = a.kv_indices + r * a.stride + p0;
  }
  // Entries 64 at a time in a VGPR, as first tiles; one that names no block gives
  // a negative tile, which is loaded as zeros and masked.
  int lreg = 0, lbase = 0;
  auto load_batch = [&](int base) {
    lbase = base;
    const int b = base + lane < cnt ? list[base + lane] : -1;
    lreg = b >= 0 && b < a.n_k ? b * SUB : -SUB;
    asm volatile("; list batch %0" ::"v"(lreg));
  };
  const int ntiles = DENSE ? cnt : cnt * SUB;
  auto fetch = [&](int j) -> int {
    if (j >= ntiles) return -1;
    if constexpr (DENSE) {
      return first + j;
    } else {
      const int e = j / SUB;
      if (e >= lbase + 64) load_batch(lbase + 64);
      return __builtin_amdgcn_readlane(lreg, e - lbase) + j % SUB;
    }
  };

  const BwdOffsets<D> off(lane);
  const TileLoad<C, NW> load(wave, lane);
  const uint16_t* const kbase = a.k + bh * a.lk * D;
  const uint16_t* const vbase = a.v + bh * a.lk * D;
  const TileRows<C> rows(a.lk);
  auto issue = [&](int tile, int slot) {
    load.issue(load.rsrc(kbase, tile, rows.bytes(tile)), ks[slot], wave);
    load.issue(load.rsrc(vbase, tile, rows.bytes(tile)), vs[slot], wave);
  };
  // keys past Lk, and all of a tile that does not exist, are masked
  auto mask_tile = [&](f32x16& x, int tile) {
    const int64_t left = tile < 0 ? 0 : a.lk - (int64_t)tile * C::KB;
    const int vis = (int)(left < 0 ? 0 : left) - 4 * hh;
    asm volatile("; mask");  // (keeps the branch around this: it is rarely taken)
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (8 * (e / 4) + e % 4 >= vis) x[e] = -INFINITY;
  };
  f32x16 acc[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;

  if (ntiles > 0) {
    // MFMA n < NA of a step: S (n even) or dP of tile t + 1; n >= NA: dQ of tile t
    auto read_a = [&](int n, int slot) -> bf16x8 {
      return tile_row<D>(n % 2 == 0 ? ks[slot] : vs[slot], off, 0, n / 2);
    };
    auto read_b = [&](int m, int slot) -> bf16x8 { return tile_col<D>(ks[slot], off, 0, m / C::DT, m % C::DT); };
    if constexpr (!DENSE) load_batch(0);
    int t0 = fetch(0), t1 = fetch(1), t2 = fetch(2);
    issue(t0, 0);
    issue(t1, 1);
    issue(t2, 2);
    wait_vmcnt<0>();
    __syncthreads();
    f32x16 s, dp = start;  // S and dP of tile t
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
    static_for<C::NA>([&](auto nc) {
      constexpr int n = decltype(nc)::value;
      const bf16x8 x = read_a(n, 0);
      if constexpr (n % 2 == 0) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, qf[n / 2], s, 0, 0, 0);
      else dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, dof[n / 2], dp, 0, 0, 0);
    });
    if ((uint32_t)t0 >= rows.whole) mask_tile(s, t0);
    bf16x8 ahead[C::P];  // operands of the next MFMAs
#pragma unroll
    for (int i = 0; i < C::P; ++i) ahead[i] = read_a(i, 1);

    int j = 0;  // tile t is the walk's j-th
    auto step = [&](auto tc) {
      constexpr int T = decltype(tc)::value;  // j mod RING: tile t's slot
      constexpr int S1 = (T + 1) % C::RING, S2 = (T + 2) % C::RING, S3 = (T + 3) % C::RING;
      constexpr int X = C::NM - C::P;         // MFMA behind which the barrier stands
      int t3;
      uint32_t bytes;
      i32x4 rk, rv;
      f32x16 sn, dn = start;
#pragma unroll
      for (int e = 0; e < 16; ++e) sn[e] = 0.f;
      bf16x8 op[C::NM + C::P];
      float x[16], p[16], ds[16];
      u32x8 pd;
#pragma unroll
      for (int i = 0; i < C::P; ++i) op[i] = ahead[i];
      auto logit = [&](auto ec) {
        constexpr int e = decltype(ec)::value;
        if constexpr (e < 16) {
          x[e] = fmaf(s[e], a.scale_log2, nl);
          asm volatile("" : "+v"(x[e]));  // holds the work here (it would otherwise sink to its uses)
        }
      };
      auto prob = [&](auto ec) {
        constexpr int e = decltype(ec)::value;
        if constexpr (e < 16) {
          p[e] = __builtin_amdgcn_exp2f(x[e]);
          asm volatile("" : "+v"(p[e]));
        }
      };
      // each stage works one element behind the stage before
      auto element = [&](auto ec) {
        constexpr int e = decltype(ec)::value;
        logit(std::integral_constant<int, e + 2>{});
        prob(std::integral_constant<int, e + 1>{});
        ds[e] = p[e] * (C::START ? dp[e] : dp[e] + nd);
        asm volatile("" : "+v"(ds[e]));
        if constexpr (e % 2 == 1) pd[e / 2] = pack2_bf16(ds[e - 1], ds[e]);
      };
      logit(std::integral_constant<int, 0>{});
      logit(std::integral_constant<int, 1>{});
      prob(std::integral_constant<int, 0>{});
      __builtin_amdgcn_sched_barrier(0);
      static_for<C::NM>([&](auto nc) {
        constexpr int n = decltype(nc)::value;
        // one wait for the operands of four MFMAs
        if constexpr (n % 4 == 0) asm volatile("" ::"v"(op[n]), "v"(op[n + 1]), "v"(op[n + 2]), "v"(op[n + 3]));
        if constexpr (n < C::NA) {
          if constexpr (n % 2 == 0) sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[n], qf[n / 2], sn, 0, 0, 0);
          else dn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[n], dof[n / 2], dn, 0, 0, 0);
        } else {
          constexpr int half = (n - C::NA) / C::DT, dt = (n - C::NA) % C::DT;
          acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[n], pack_half(pd, half), acc[dt], 0, 0, 0);
        }
        // The scalar work of tile t + 3's loads is spread over the MFMAs before the
        // barrier, the loads over those behind it: in one place they hold up the wave.
        if constexpr (n == X - 6) t3 = fetch(j + 3);
        if constexpr (n == X - 4) bytes = rows.bytes(t3);
        if constexpr (n == X - 3) rk = load.rsrc(kbase, t3, bytes);
        if constexpr (n == X - 2) rv = load.rsrc(vbase, t3, bytes);
        if constexpr (n == X) {
          publish();
          load.issue(rk, ks[S3], wave);
        }
        if constexpr (n == X + 1) load.issue(rv, vs[S3], wave);
        constexpr int r = n + C::P;  // the operand to read now
        if constexpr (r < C::NA) op[r] = read_a(r, S1);
        else if constexpr (r < C::NM) op[r] = read_b(r - C::NA, T);
        else op[r] = read_a(r - C::NM, S2);
        // the elements whose turn it is
        constexpr int e0 = (n * 16 + C::SPREAD - 1) / C::SPREAD;
        static_for<2>([&](auto k) {
          constexpr int e = e0 + decltype(k)::value;
          if constexpr (e < 16 && e * C::SPREAD / 16 == n) element(std::integral_constant<int, e>{});
        });
        __builtin_amdgcn_sched_barrier(0);
      });
#pragma unroll
      for (int i = 0; i < C::P; ++i) ahead[i] = op[C::NM + i];
      s = sn;
      dp = dn;
      t0 = t1;
      t1 = t2;
      t2 = t3;
      if ((uint32_t)t0 >= rows.whole) mask_tile(s, t0);
    };
    while (true) {
      step(std::integral_constant<int, 0>{});
      if (++j >= ntiles) break;
      step(std::integral_constant<int, 1>{});
      if (++j >= ntiles) break;
      step(std::integral_constant<int, 2>{});
      if (++j >= ntiles) break;
      step(std::integral_constant<int, 3>{});
      if (++j >= ntiles) break;
    }
    wait_vmcnt<0>();  // loads past the end of the list still write LDS
  }
  if (!row_ok) return;
  if (a.dq_ranges > 1) {
    float* out = a.part + ((int64_t)range * a.bh * a.lq + bh * a.lq + row) * D + 4 * hh;
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(out + 32 * t + 8 * g) =
            make_float4(acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]);
  } else {
    uint16_t* out = a.dq + (bh * a.lq + row) * D + 4 * hh;
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<uint2*>(out + 32 * t + 8 * g) =
            make_uint2(pack2_bf16(acc[t][4 * g] * a.scale, acc[t][4 * g + 1] * a.scale),
                       pack2_bf16(acc[t][4 * g + 2] * a.scale, acc[t][4 * g + 3] * a.scale));
  }
}

// ---- dK and dV: one work-group per (head, query range, key group of 32 NW keys),
// one wave per 32 keys.  Per 32-query sub-tile S = Q K^T and dP = dO V^T (lane: 16
// queries of one key), then dV^T += dO^T P and dK^T += Q^T dS.
//
// Step t holds S and dP of tile t + 1, then dV and dK of tile t: 32 MFMAs at D = 128,
// 16 at 64.  The softmax of tile t is spread over the first two thirds of them, each
// element behind one MFMA, and each MFMA's operand is read from LDS P MFMAs earlier.
// S starts from -lse / s and dP from -delta, so an element takes a product, an
// exponential, a product and its packing.  A tile lands in LDS a whole step before its
// first read, and one barrier per step both publishes it and frees the slot of tile
// t - 1.
//
// At D = 128 the sums, the wave's K and V and the operands in flight take some 350
// registers, so one wave runs per SIMD.  It issues one instruction per 5 cycles at
// most, so what a step costs is its count of instructions (the first form of this step,
// with 340 of them, kept the matrix cores busy 48% of the time, LDS at a quarter of its
// rate).
template <int D>
struct DkvCfg : BwdCfg<D> {
  using B = BwdCfg<D>;
  static constexpr int NA = 2 * B::DS, NB = 4 * B::DT, NM = NA + NB;  // MFMAs of a step
  static constexpr int SPREAD = NM * 11 / 16;      // MFMAs that the softmax is spread over
  static constexpr int P = 6;                      // MFMAs between an operand's read and its use
  static constexpr int RING = 4;                   // tiles in LDS, Q and dO each
  static constexpr int WAVES = D == 128 ? 1 : 2;   // per SIMD
};

template <int D>
struct alignas(1024) DkvLds {
  uint16_t qs[DkvCfg<D>::RING][DkvCfg<D>::TILE], dos[DkvCfg<D>::RING][DkvCfg<D>::TILE];
  float st[DkvCfg<D>::RING][64];
};

template <int D, int NW, bool DENSE>
__device__ __forceinline__ void attn_bwd_dkv(const BwdArgs& a, DkvLds<D>& lds, uint32_t index, uint32_t groups) {
  using C = DkvCfg<D>;
  constexpr int KEYS = 32 * NW, SUB = KEYS / C::KB;  // (sparse: a query block is SUB tiles)
  auto& qs = lds.qs;
  auto& dos = lds.dos;
  auto& st = lds.st;
  const int64_t n_g = (a.lk + KEYS - 1) / KEYS;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int l32 = lane % 32, hh = lane / 32;
  // Key blocks that far more queries list than the average (forced ones: all of them) come
  // first: begun last they would run on alone.
  // (The grid holds the pieces, as many as there can be, and every block; a block among the
  // pieces returns here, and so do work-groups past the end.)
  int slot = -1, range = 0, ranges = a.dkv_ranges, kg;
  int b0 = 0, b1 = a.n_q;  // (sparse) the query blocks that the walk is about
  int64_t bh;
  if (!DENSE && a.list_min > 0) {
    const int first = __builtin_amdgcn_readfirstlane(*a.piece_count);
    int item = (int)index - first;
    if (item < 0) {
      const BwdPiece p = a.pieces[index];
      item = __builtin_amdgcn_readfirstlane(p.block);
      ranges = __builtin_amdgcn_readfirstlane(p.pieces);
      slot = __builtin_amdgcn_readfirstlane(p.slot);
      b0 = __builtin_amdgcn_readfirstlane(p.begin);
      b1 = __builtin_amdgcn_readfirstlane(p.end);
    } else if (item >= a.bh * (int)n_g || __builtin_amdgcn_readfirstlane((int)a.listed[item]) != 0) {
      return;
    }
    bh = item / (int)n_g;
    kg = item - (int)bh * (int)n_g;
  } else {
    const int64_t w = DENSE ? xcd_linear(index, groups) : index;
    const int64_t pair = w / n_g;
    kg = (int)(w - pair * n_g);
    bh = pair / ranges;
    range = (int)(pair - bh * ranges);
  }

  const int64_t key = (int64_t)kg * KEYS + wave * 32 + l32;
  const bool key_ok = key < a.lk;
  bf16x8 kf[C::DS], vf[C::DS];
  {
    const int64_t at = (bh * a.lk + (key_ok ? key : 0)) * D + 8 * hh;
#pragma unroll
    for (int s = 0; s < C::DS; ++s) {
      kf[s] = load_row(a.k + at + 16 * s, key_ok);
      vf[s] = load_row(a.v + at + 16 * s, key_ok);
    }
  }

  // The walk: query tiles in ascending order.  Sparse: the set bits of the key
  // block's words, 64 words at a time in a VGPR.
  const uint32_t* words = nullptr;
  int wpos, wend;            // words (dense: tiles) still to load, end of the range
  uint32_t wreg = 0, cur = 0;
  uint64_t full = 0;         // words of the batch that have bits left
  int wbase = 0, qb32 = 0, sub = SUB, blk = 0;
  if constexpr (DENSE) {
    const int64_t n = (a.lq + C::KB - 1) / C::KB;
    wpos = (int)(n * range / ranges);
    wend = (int)(n * (range + 1) / ranges);
  } else {
    words = a.bits + (bh * a.n_k + kg) * a.n_words;
    wpos = b0 / 32;
    wend = (b1 + 31) / 32;
  }
  auto next_tile = [&]() -> int {  // -1: none is left
    if constexpr (DENSE) {
      return wpos < wend ? wpos++ : -1;
    } else {
      if (sub == SUB) {
        if (cur == 0) {
          while (full == 0) {
            if (wpos >= wend) return -1;
            wbase = wpos;
            wreg = wpos + lane < wend ? words[wpos + lane] : 0u;
            const int first = (wpos + lane) * 32, last = first + 32;
            if (first < b0) wreg &= ~0u << (b0 - first);
            if (last > b1 && wreg != 0) wreg &= ~0u >> (last - b1);
            full = __builtin_amdgcn_ballot_w64(wreg != 0);
            wpos += 64;
          }
          const int i = __builtin_ctzll(full);
          full &= full - 1;
          cur = (uint32_t)__builtin_amdgcn_readlane((int)wreg, i);
          qb32 = (wbase + i) * 32;
        }
        blk = qb32 + __builtin_ctz(cur);
        cur &= cur - 1;
        sub = 0;
      }
      return blk * SUB + sub++;
    }
  };

  const BwdOffsets<D> off(lane);
  const TileLoad<C, NW> load(wave, lane);
  const uint16_t* const qbase = a.q + bh * a.lq * D;
  const uint16_t* const dobase = a.d_o + bh * a.lq * D;
  const float* const stbase = a.stats + bh * a.n_q * a.block * 2;
  const TileRows<C> rows(a.lq);
  auto issue = [&](int tile, int slot) {
    load.issue(load.rsrc(qbase, tile, rows.bytes(tile)), qs[slot], wave);
    load.issue(load.rsrc(dobase, tile, rows.bytes(tile)), dos[slot], wave);
    // (every wave loads the same statistics, so that all wait for as many loads)
    dma_floats(raw_rsrc(stbase + (int64_t)tile * 64, tile < 0 ? 0u : 256u), st[slot], lane);
  };

  f32x16 dk[C::DT], dv[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) dk[t][e] = dv[t][e] = 0.f;

  int t0 = next_tile();
  if (t0 >= 0) {
    // MFMA n < NA of a step: S (n even) or dP of tile t + 1; n >= NA: dV or dK of tile t
    auto read_a = [&](int n, int slot) -> bf16x8 {
      return tile_row<D>(n % 2 == 0 ? qs[slot] : dos[slot], off, 0, n / 2);
    };
    auto read_b = [&](int m, int slot) -> bf16x8 {
      return tile_col<D>(m % 2 == 0 ? dos[slot] : qs[slot], off, 0, m / (2 * C::DT), m / 2 % C::DT);
    };
    // where S and dP start from: element e is row 8 (e / 4) + 4 h + e % 4
    auto read_init = [&](int g, int slot, f32x16& x, f32x16& y) {
      const f32x4 l = *reinterpret_cast<const f32x4*>(st[slot] + 8 * g + 4 * hh);
      const f32x4 d = *reinterpret_cast<const f32x4*>(st[slot] + 32 + 8 * g + 4 * hh);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[4 * g + e] = l[e];
        y[4 * g + e] = d[e];
      }
    };
    f32x16 s, dp;        // S and dP of tile t
    f32x16 s1, dp1;      // the start of those of tile t + 1
    bf16x8 ahead[C::P];  // operands of the next MFMAs

    int t1 = next_tile(), t2 = next_tile();
    issue(t0, 0);
    issue(t1, 1);
    issue(t2, 2);
    wait_vmcnt<0>();
    __syncthreads();
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      read_init(g, 0, s, dp);
      read_init(g, 1, s1, dp1);
    }
    static_for<C::NA>([&](auto nc) {
      constexpr int n = decltype(nc)::value;
      const bf16x8 x = read_a(n, 0);
      if constexpr (n % 2 == 0) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, kf[n / 2], s, 0, 0, 0);
      else dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, vf[n / 2], dp, 0, 0, 0);
    });
#pragma unroll
    for (int i = 0; i < C::P; ++i) ahead[i] = read_a(i, 1);

    auto step = [&](auto tc) {
      constexpr int T = decltype(tc)::value;  // t mod RING: tile t's slot
      constexpr int S1 = (T + 1) % C::RING, S2 = (T + 2) % C::RING, S3 = (T + 3) % C::RING;
      constexpr int X = C::NM - C::P;         // MFMA behind which the barrier stands
      int t3;
      uint32_t bytes;
      i32x4 rq, rdo, rst;
      f32x16 sn = s1, dn = dp1;
      bf16x8 op[C::NM + C::P];
      float x[16], p[16], ds[16];
      u32x8 pp, pd;
#pragma unroll
      for (int i = 0; i < C::P; ++i) op[i] = ahead[i];
      auto logit = [&](auto ec) {
        constexpr int e = decltype(ec)::value;
        if constexpr (e < 16) {
          x[e] = s[e] * a.scale_log2;
          asm volatile("" : "+v"(x[e]));  // holds the work here (it would otherwise sink to its uses)
        }
      };
      auto prob = [&](auto ec) {
        constexpr int e = decltype(ec)::value;
        if constexpr (e < 16) {
          p[e] = __builtin_amdgcn_exp2f(x[e]);
          asm volatile("" : "+v"(p[e]));
        }
      };
      // each stage works one element behind the stage before
      auto element = [&](auto ec) {
        constexpr int e = decltype(ec)::value;
        logit(std::integral_constant<int, e + 2>{});
        prob(std::integral_constant<int, e + 1>{});
        ds[e] = p[e] * dp[e];
        asm volatile("" : "+v"(ds[e]));
        if constexpr (e % 2 == 1) {
          pp[e / 2] = pack2_bf16(p[e - 1], p[e]);
          pd[e / 2] = pack2_bf16(ds[e - 1], ds[e]);
        }
      };
      logit(std::integral_constant<int, 0>{});
      logit(std::integral_constant<int, 1>{});
      prob(std::integral_constant<int, 0>{});
      __builtin_amdgcn_sched_barrier(0);
      static_for<C::NM>([&](auto nc) {
        constexpr int n = decltype(nc)::value;
        // one wait for the operands of four MFMAs
        if constexpr (n % 4 == 0) asm volatile("" ::"v"(op[n]), "v"(op[n + 1]), "v"(op[n + 2]), "v"(op[n + 3]));
        if constexpr (n < C::NA) {
          if constexpr (n % 2 == 0) sn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[n], kf[n / 2], sn, 0, 0, 0);
          else dn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[n], vf[n / 2], dn, 0, 0, 0);
        } else {
          constexpr int m = n - C::NA, half = m / (2 * C::DT), dt = m / 2 % C::DT;
          if constexpr (m % 2 == 0)
            dv[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[n], pack_half(pp, half), dv[dt], 0, 0, 0);
          else
            dk[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[n], pack_half(pd, half), dk[dt], 0, 0, 0);
        }
        if constexpr (n == X - 6) t3 = next_tile();
        if constexpr (n == X - 4) bytes = rows.bytes(t3);
        if constexpr (n == X - 3) rq = load.rsrc(qbase, t3, bytes);
        if constexpr (n == X - 2) rdo = load.rsrc(dobase, t3, bytes);
        if constexpr (n == X - 1) rst = raw_rsrc(stbase + (int64_t)t3 * 64, t3 < 0 ? 0u : 256u);
        if constexpr (n == X) {
          publish();
          load.issue(rq, qs[S3], wave);
        }
        if constexpr (n == X + 1) load.issue(rdo, dos[S3], wave);
        if constexpr (n == X + 2) dma_floats(rst, st[S3], lane);
        constexpr int r = n + C::P;  // the operand to read now
        if constexpr (r < C::NA) op[r] = read_a(r, S1);
        else if constexpr (r < C::NM) op[r] = read_b(r - C::NA, T);
        else op[r] = read_a(r - C::NM, S2);
        if constexpr (n >= C::NM - 4) read_init(n - (C::NM - 4), S2, s1, dp1);
        // the elements whose turn it is
        constexpr int e0 = (n * 16 + C::SPREAD - 1) / C::SPREAD;
        static_for<2>([&](auto k) {
          constexpr int e = e0 + decltype(k)::value;
          if constexpr (e < 16 && e * C::SPREAD / 16 == n) element(std::integral_constant<int, e>{});
        });
        __builtin_amdgcn_sched_barrier(0);
      });
#pragma unroll
      for (int i = 0; i < C::P; ++i) ahead[i] = op[C::NM + i];
      s = sn;
      dp = dn;
      t0 = t1;
      t1 = t2;
      t2 = t3;
    };
    while (true) {
      step(std::integral_constant<int, 0>{});
      if (t0 < 0) break;
      step(std::integral_constant<int, 1>{});
      if (t0 < 0) break;
      step(std::integral_constant<int, 2>{});
      if (t0 < 0) break;
      step(std::integral_constant<int, 3>{});
      if (t0 < 0) break;
    }
    wait_vmcnt<0>();  // loads past the end of the walk still write LDS
  }
  if (!key_ok) return;
  const int64_t at = (bh * a.lk + key) * D + 4 * hh;
  // partial results: of whole tensors, or of a piece
  const int64_t all = slot < 0 ? (int64_t)a.bh * a.lk * D : (int64_t)KEYS * D;
  float* const part = slot < 0 ? a.part_kv + range * 2 * all + at
                               : a.part_piece + slot * 2 * all + (wave * 32 + l32) * D + 4 * hh;
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int64_t o = 32 * t + 8 * g;
      const f32x16 &x = dk[t], &y = dv[t];
      if (ranges > 1) {
        *reinterpret_cast<float4*>(part + o) = make_float4(x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]);
        *reinterpret_cast<float4*>(part + all + o) = make_float4(y[4 * g], y[4 * g + 1], y[4 * g + 2], y[4 * g + 3]);
      } else {
        *reinterpret_cast<uint2*>(a.dk + at + o) =
            make_uint2(pack2_bf16(x[4 * g] * a.scale, x[4 * g + 1] * a.scale),
                       pack2_bf16(x[4 * g + 2] * a.scale, x[4 * g + 3] * a.scale));
        *reinterpret_cast<uint2*>(a.dv + at + o) =
            make_uint2(pack2_bf16(y[4 * g], y[4 * g + 1]), pack2_bf16(y[4 * g + 2], y[4 * g + 3]));
      }
    }
}

template <int D, int NW, bool DENSE>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attn_bwd_dq_kernel(BwdArgs a) {
  __shared__ DqLds<D> lds;
  attn_bwd_dq<D, NW, DENSE>(a, lds, blockIdx.x, gridDim.x);
}

template <int D, int NW, bool DENSE>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(DkvCfg<D>::WAVES, DkvCfg<D>::WAVES)))
void attn_bwd_dkv_kernel(BwdArgs a) {
  __shared__ DkvLds<D> lds;
  attn_bwd_dkv<D, NW, DENSE>(a, lds, blockIdx.x, gridDim.x);
}

// Both passes in one launch, for calls of up to two waves per SIMD: neither waits for the
// other's last work-group.  At D = 128 dQ gives up its second wave per SIMD for it, so calls
// of many rounds keep their launches.  Two heads of 512 x 1,152, D = 64: 16.9 us, in two
// launches 25.5; 4 heads of 1,024 x 3,000 at 25%: 37.3 and 47.7; 8 heads: 53.4 and 59.2.
constexpr int kBothWaves = 2048;
template <int D, int NW, bool DENSE>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(DkvCfg<D>::WAVES, DkvCfg<D>::WAVES)))
void attn_bwd_both_kernel(BwdArgs a, uint32_t dq_groups) {
  __shared__ union {
    DqLds<D> dq;
    DkvLds<D> dkv;
  } lds;
  if (blockIdx.x < dq_groups) attn_bwd_dq<D, NW, DENSE>(a, lds.dq, blockIdx.x, dq_groups);
  else attn_bwd_dkv<D, NW, DENSE>(a, lds.dkv, blockIdx.x - dq_groups, gridDim.x - dq_groups);
}

// ---- sums the ranges' partial results, in order: out = bf16(scale * sum_r part[r])
__global__ __launch_bounds__(256) void attn_bwd_sum_kernel(const float* part, int64_t stride, int ranges, int64_t n,
                                                           float scale, uint16_t* out) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
  for (int r = 0; r < ranges; ++r) {
    const float4 u = *reinterpret_cast<const float4*>(part + r * stride + i);
    const float4 v = *reinterpret_cast<const float4*>(part + r * stride + i + 4);
    x.x += u.x, x.y += u.y, x.z += u.z, x.w += u.w;
    y.x += v.x, y.y += v.y, y.z += v.z, y.w += v.w;
  }
  *reinterpret_cast<uint4*>(out + i) =
      make_uint4(pack2_bf16(x.x * scale, x.y * scale), pack2_bf16(x.z * scale, x.w * scale),
                 pack2_bf16(y.x * scale, y.y * scale), pack2_bf16(y.z * scale, y.w * scale));
}

// ---- the same for key blocks that were cut, an eighth of a block's dK and dV at a time
constexpr int kPieceSumGroups = 2048;
template <int D>
__global__ __launch_bounds__(256) void attn_bwd_piece_sum_kernel(BwdArgs a) {
  const int n = *a.piece_count, all = a.block * D;
  for (int w = blockIdx.x; w < 8 * n; w += kPieceSumGroups) {
    const BwdPiece p = a.pieces[w / 8];
    if (p.piece != 0 || p.pieces <= 1) continue;  // (a block's first piece stands for it)
    const int64_t bh = p.block / a.n_k, kg = p.block - bh * a.n_k, left = a.lk - kg * a.block;
    const float* part = a.part_piece + (int64_t)p.slot * 2 * all;
    const int valid = (int)(left < a.block ? left : a.block) * D;
    for (int i = (w % 8 * 256 + threadIdx.x) * 4; i < 2 * all; i += 8 * 256 * 4) {
      const bool is_v = i >= all;
      const int at = is_v ? i - all : i;
      if (at >= valid) continue;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int r = 0; r < p.pieces; ++r) {
        const float4 u = *reinterpret_cast<const float4*>(part + (int64_t)r * 2 * all + i);
        x.x += u.x, x.y += u.y, x.z += u.z, x.w += u.w;
      }
      const float s = is_v ? 1.f : a.scale;
      uint16_t* out = (is_v ? a.dv : a.dk) + (bh * a.lk + kg * a.block) * D + at;
      *reinterpret_cast<uint2*>(out) = make_uint2(pack2_bf16(x.x * s, x.y * s), pack2_bf16(x.z * s, x.w * s));
    }
  }
}

template <int D, int NW, bool DENSE>
static hipError_t launch_passes(const BwdArgs& a, hipStream_t stream) {
  constexpr int ROWS = 32 * NW;
  const int64_t nq = (int64_t)a.bh * a.lq * D, nk = (int64_t)a.bh * a.lk * D;
  auto sum = [&](const float* part, int64_t stride, int ranges, int64_t n, float scale, uint16_t* out) {
    attn_bwd_sum_kernel<<<(n / 8 + 255) / 256, 256, 0, stream>>>(part, stride, ranges, n, scale, out);
  };
  const int64_t dq_grid = (int64_t)a.bh * a.dq_ranges * ((a.lq + ROWS - 1) / ROWS);
  const int64_t dkv_grid = (int64_t)a.bh * a.dkv_ranges * ((a.lk + ROWS - 1) / ROWS);
  if ((dq_grid + dkv_grid) * NW <= kBothWaves) {
    attn_bwd_both_kernel<D, NW, DENSE><<<dq_grid + dkv_grid + a.most_pieces, 64 * NW, 0, stream>>>(a, (uint32_t)dq_grid);
  } else {
    if (dq_grid > 0) attn_bwd_dq_kernel<D, NW, DENSE><<<dq_grid, 64 * NW, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    attn_bwd_dkv_kernel<D, NW, DENSE><<<dkv_grid + a.most_pieces, 64 * NW, 0, stream>>>(a);
  }
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (a.dq_ranges > 1) sum(a.part, nq, a.dq_ranges, nq, a.scale, a.dq);
  if (a.list_min > 0 && a.piece_max < a.n_q) attn_bwd_piece_sum_kernel<D><<<kPieceSumGroups, 256, 0, stream>>>(a);
  if (a.dkv_ranges > 1) {
    sum(a.part_kv, 2 * nk, a.dkv_ranges, nk, a.scale, a.dk);
    sum(a.part_kv + nk, 2 * nk, a.dkv_ranges, nk, 1.f, a.dv);
  }
  return hipGetLastError();
}

template <int D>
static hipError_t launch_bwd(const BwdArgs& a, bool dense, hipStream_t stream) {
  constexpr int RPW = 256 / (D / 8);
  const int64_t stat_groups = ((int64_t)a.bh * a.n_q * a.block + RPW - 1) / RPW;
  const int chunks = (a.n_k + kBitsChunk - 1) / kBitsChunk;
  const int64_t grid = stat_groups + (dense ? 0 : (int64_t)a.bh * a.n_words * chunks);
  if (grid > 0) attn_bwd_prepare_kernel<D><<<grid, 256, 0, stream>>>(a, stat_groups, chunks);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (a.list_min > 0) {
    attn_bwd_pieces_kernel<<<((int64_t)a.bh * a.n_k + 31) / 32, 256, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (dense) return launch_passes<D, 4, true>(a, stream);
  return a.block == 64 ? launch_passes<D, 2, false>(a, stream) : launch_passes<D, 4, false>(a, stream);
}

hipError_t launch_attn_bwd(const BwdArgs& a, int d, bool dense, hipStream_t stream) {
  return d == 128 ? launch_bwd<128>(a, dense, stream) : launch_bwd<64>(a, dense, stream);
}

}  // namespace sparstar
