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
#include "attn_device.h"

namespace sparstar {

// Tiles are 8 KB: 32 rows at D = 128, 64 at D = 64.  Rows are stored unpadded in LDS
// and their 16-byte chunks XOR-permuted by swz(row), which leaves both reads of a
// tile free of bank conflicts: 16 consecutive rows of one chunk (ds_read_b128), and
// four consecutive rows of four chunks (the transpose read).
template <int D>
struct BwdCfg {
  static constexpr int KB = attn_tile_keys(D);  // rows per tile
  static constexpr int KT = KB / 32;            // 32-row sub-tiles
  static constexpr int DS = D / 16;             // MFMA k-steps over D
  static constexpr int DT = D / 32;             // 32-row tiles of a D-row result
  static constexpr int RB = D * 2;              // bytes per row
  static constexpr int CPR = D / 8;             // 16-byte chunks per row
  static constexpr int RPD = 1024 / RB;         // rows per direct-to-LDS wave load
  static constexpr int TILE = KB * D;           // elements per tile
  static constexpr int TILE_BYTES = TILE * 2;
  static_assert(TILE_BYTES == 8192, "8 KB tiles");
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

// The direct-to-LDS loads of one tile by NW waves.
template <int D, int NW>
struct TileLoad {
  using C = BwdCfg<D>;
  static constexpr int N = 8 / NW;  // 1 KB loads per wave
  uint32_t off[N];
  __device__ __forceinline__ TileLoad(int wave, int lane) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = C::RPD * (N * wave + i) + lane / C::CPR;
      // (the instruction adds 1024 i)
      off[i] = (uint32_t)(r * C::RB + 16 * ((lane % C::CPR) ^ bwd_swz<D>(r)) - 1024 * i);
    }
  }
  // rows [row0, row0 + KB) of a [rows, D] tensor; rows past its end arrive as zeros
  __device__ __forceinline__ void issue(const uint16_t* base, int64_t row0, int64_t rows, uint16_t* slot,
                                        int wave) const {
    int64_t left = rows - row0;
    left = left < 0 ? 0 : (left > C::KB ? C::KB : left);
    const i32x4 rs = raw_rsrc(base + row0 * D, (uint32_t)left * (uint32_t)C::RB);
    dma_tile<N>(lds_addr(slot) + (uint32_t)(N * wave) * 1024u, off, rs);
  }
};

// 64 consecutive floats into LDS (lane l: 4 bytes at +4 l)
__device__ __forceinline__ void dma_floats(const float* src, float* slot, int lane) {
  const i32x4 rs = raw_rsrc(src, 256);
  const uint32_t voff = (uint32_t)lane * 4u;
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "buffer_load_dword %1, %2, 0 offen lds"
      :
      : "s"(lds_addr(slot)), "v"(voff), "s"(rs)
      : "memory", "m0");
}

// ---- per-row statistics.  Rows are kept in groups of 32, [32] of
// -lse log2(e) then [32] of -delta, padded to whole query blocks: a row past Lq,
// and one that saw no key, gets -inf and 0, which makes its P and dS zero.
template <int D>
__global__ __launch_bounds__(256) void attn_bwd_stats_kernel(BwdArgs a) {
  constexpr int LPR = D / 8, RPW = 256 / LPR;
  const int64_t rows_pad = (int64_t)a.n_q * a.block;
  const int64_t i = (int64_t)blockIdx.x * RPW + threadIdx.x / LPR;
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
        nl = -l * 1.44269504088896340736f;
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
constexpr int kBitsChunk = 8192;
__global__ __launch_bounds__(1024) void attn_bwd_bits_kernel(BwdArgs a) {
  __shared__ uint32_t bits[kBitsChunk];
  const int64_t bh = blockIdx.x / a.n_words;
  const int word = (int)(blockIdx.x - bh * a.n_words);
  const int lo = (int)blockIdx.y * kBitsChunk;
  const int hi = a.n_k - lo < kBitsChunk ? a.n_k : lo + kBitsChunk;
  for (int j = threadIdx.x; j < hi - lo; j += 1024) bits[j] = 0u;
  __syncthreads();
  const int lane = threadIdx.x % 64;
  for (int i = threadIdx.x / 64; i < 32; i += 16) {
    const int qb = 32 * word + i;
    if (qb >= a.n_q) break;
    const int64_t r = bh * a.n_q + qb;
    int n = a.kv_num_blocks[r];
    n = n < 0 ? 0 : (n > a.stride ? a.stride : n);
    for (int e = lane; e < n; e += 64) {
      const int j = a.kv_indices[r * a.stride + e];
      if (j >= lo && j < hi) atomicOr(&bits[j - lo], 1u << i);
    }
  }
  __syncthreads();
  for (int j = threadIdx.x; j < hi - lo; j += 1024) a.bits[(bh * a.n_k + lo + j) * a.n_words + word] = bits[j];
}

// ---- dQ: one work-group per (head, list range, query group of 32 NW rows), one
// wave per 32 rows.  Per 32-key sub-tile S^T = K Q^T and dP^T = V dO^T (lane: 16
// keys of one query), then dQ^T += K^T dS^T with dS rounded to bf16 once.
template <int D, int NW, bool DENSE>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2)))
void attn_bwd_dq_kernel(BwdArgs a) {
  using C = BwdCfg<D>;
  constexpr int ROWS = 32 * NW, SUB = ROWS / C::KB;  // (sparse: a list entry is SUB tiles)
  __shared__ __attribute__((aligned(1024))) uint16_t ks[2][C::TILE];
  __shared__ __attribute__((aligned(1024))) uint16_t vs[2][C::TILE];
  const int64_t n_g = (a.lq + ROWS - 1) / ROWS;
  const int64_t w = xcd_linear(blockIdx.x, gridDim.x);
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
  float nl = -INFINITY, nd = 0.f;
  if (row_ok) {
    const int64_t i = bh * a.n_q * a.block + row;
    nl = a.stats[(i / 32) * 64 + i % 32];
    nd = a.stats[(i / 32) * 64 + 32 + i % 32];
  }

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
    if constexpr (DENSE) {
      return first + j;
    } else {
      const int e = j / SUB;
      if (e >= lbase + 64) load_batch(lbase + 64);
      return __builtin_amdgcn_readlane(lreg, e - lbase) + j % SUB;
    }
  };

  const BwdOffsets<D> off(lane);
  const TileLoad<D, NW> load(wave, lane);
  const uint16_t* const kbase = a.k + bh * a.lk * D;
  const uint16_t* const vbase = a.v + bh * a.lk * D;
  auto issue = [&](int tile, int slot) {
    const int64_t row0 = tile < 0 ? 0 : (int64_t)tile * C::KB, rows = tile < 0 ? 0 : a.lk;
    load.issue(kbase, row0, rows, ks[slot], wave);
    load.issue(vbase, row0, rows, vs[slot], wave);
  };
  f32x16 acc[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;

  if (ntiles > 0) {
    if constexpr (!DENSE) load_batch(0);
    int tile = fetch(0);
    issue(tile, 0);
    for (int j = 0; j < ntiles; ++j) {
      const int next = j + 1 < ntiles ? fetch(j + 1) : -1;
      wait_vmcnt<0>();
      __syncthreads();
      if (j + 1 < ntiles) issue(next, (j + 1) & 1);
      const uint16_t* kt_lds = ks[j & 1];
      const uint16_t* vt_lds = vs[j & 1];
      const int64_t left = tile < 0 ? 0 : a.lk - (int64_t)tile * C::KB;
#pragma unroll
      for (int kt = 0; kt < C::KT; ++kt) {
        f32x16 s, dp;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[e] = 0.f;
          dp[e] = nd;
        }
#pragma unroll
        for (int i = 0; i < C::DS; ++i) {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_row<D>(kt_lds, off, kt, i), qf[i], s, 0, 0, 0);
          dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_row<D>(vt_lds, off, kt, i), dof[i], dp, 0, 0, 0);
        }
        if (left < C::KB) {
          const int vis = (int)left - 32 * kt - 4 * hh;
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (8 * (e / 4) + e % 4 >= vis) s[e] = -INFINITY;
        }
        u32x8 pk;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[e], a.scale_log2, nl));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(s[e + 1], a.scale_log2, nl));
          pk[e / 2] = pack2_bf16(p0 * dp[e], p1 * dp[e + 1]);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int t = 0; t < C::DT; ++t)
            acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_col<D>(kt_lds, off, kt, half, t),
                                                             pack_half(pk, half), acc[t], 0, 0, 0);
      }
      tile = next;
    }
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
// queries of one key), then dV^T += dO^T P and dK^T += Q^T dS.  The sums and the
// wave's K and V take 192 registers at D = 128, so one wave runs per SIMD there.
template <int D, int NW, bool DENSE>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(D == 128 ? 1 : 2, D == 128 ? 1 : 2)))
void attn_bwd_dkv_kernel(BwdArgs a) {
  using C = BwdCfg<D>;
  constexpr int KEYS = 32 * NW, SUB = KEYS / C::KB;  // (sparse: a query block is SUB tiles)
  __shared__ __attribute__((aligned(1024))) uint16_t qs[2][C::TILE];
  __shared__ __attribute__((aligned(1024))) uint16_t dos[2][C::TILE];
  __shared__ __attribute__((aligned(1024))) float st[2][64 * C::KT];
  const int64_t n_g = (a.lk + KEYS - 1) / KEYS;
  const int64_t w = xcd_linear(blockIdx.x, gridDim.x);
  const int64_t pair = w / n_g;
  const int kg = (int)(w - pair * n_g);
  const int64_t bh = pair / a.dkv_ranges;
  const int range = (int)(pair - bh * a.dkv_ranges);
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int l32 = lane % 32, hh = lane / 32;

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
    wpos = (int)(n * range / a.dkv_ranges);
    wend = (int)(n * (range + 1) / a.dkv_ranges);
  } else {
    words = a.bits + (bh * a.n_k + kg) * a.n_words;
    wpos = (int)((int64_t)a.n_words * range / a.dkv_ranges);
    wend = (int)((int64_t)a.n_words * (range + 1) / a.dkv_ranges);
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
  const TileLoad<D, NW> load(wave, lane);
  const uint16_t* const qbase = a.q + bh * a.lq * D;
  const uint16_t* const dobase = a.d_o + bh * a.lq * D;
  const float* const stbase = a.stats + bh * a.n_q * a.block * 2;
  auto issue = [&](int tile, int slot) {
    load.issue(qbase, (int64_t)tile * C::KB, a.lq, qs[slot], wave);
    load.issue(dobase, (int64_t)tile * C::KB, a.lq, dos[slot], wave);
    if (wave < C::KT) dma_floats(stbase + ((int64_t)tile * C::KT + wave) * 64, st[slot] + 64 * wave, lane);
  };
  f32x16 dk[C::DT], dv[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) dk[t][e] = dv[t][e] = 0.f;

  int tile = next_tile();
  if (tile >= 0) issue(tile, 0);
  for (int j = 0; tile >= 0; ++j) {
    const int next = next_tile();
    wait_vmcnt<0>();
    __syncthreads();
    if (next >= 0) issue(next, (j + 1) & 1);
    const uint16_t* qt = qs[j & 1];
    const uint16_t* dt = dos[j & 1];
    const float* stt = st[j & 1];
#pragma unroll
    for (int kt = 0; kt < C::KT; ++kt) {
      f32x16 s, dp, nl;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float4 l = *reinterpret_cast<const float4*>(stt + 64 * kt + 8 * g + 4 * hh);
        const float4 d = *reinterpret_cast<const float4*>(stt + 64 * kt + 32 + 8 * g + 4 * hh);
        nl[4 * g] = l.x, nl[4 * g + 1] = l.y, nl[4 * g + 2] = l.z, nl[4 * g + 3] = l.w;
        dp[4 * g] = d.x, dp[4 * g + 1] = d.y, dp[4 * g + 2] = d.z, dp[4 * g + 3] = d.w;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
      for (int i = 0; i < C::DS; ++i) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_row<D>(qt, off, kt, i), kf[i], s, 0, 0, 0);
        dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_row<D>(dt, off, kt, i), vf[i], dp, 0, 0, 0);
      }
      u32x8 pp, pd;
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[e], a.scale_log2, nl[e]));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(s[e + 1], a.scale_log2, nl[e + 1]));
        pp[e / 2] = pack2_bf16(p0, p1);
        pd[e / 2] = pack2_bf16(p0 * dp[e], p1 * dp[e + 1]);
      }
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int t = 0; t < C::DT; ++t) {
          dv[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_col<D>(dt, off, kt, half, t), pack_half(pp, half), dv[t],
                                                          0, 0, 0);
          dk[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(tile_col<D>(qt, off, kt, half, t), pack_half(pd, half), dk[t],
                                                          0, 0, 0);
        }
    }
    tile = next;
  }
  if (!key_ok) return;
  const int64_t at = (bh * a.lk + key) * D + 4 * hh, all = (int64_t)a.bh * a.lk * D;
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int64_t o = at + 32 * t + 8 * g;
      const f32x16 &x = dk[t], &y = dv[t];
      if (a.dkv_ranges > 1) {
        float* part = a.part + (int64_t)range * 2 * all;
        *reinterpret_cast<float4*>(part + o) = make_float4(x[4 * g], x[4 * g + 1], x[4 * g + 2], x[4 * g + 3]);
        *reinterpret_cast<float4*>(part + all + o) = make_float4(y[4 * g], y[4 * g + 1], y[4 * g + 2], y[4 * g + 3]);
      } else {
        *reinterpret_cast<uint2*>(a.dk + o) = make_uint2(pack2_bf16(x[4 * g] * a.scale, x[4 * g + 1] * a.scale),
                                                         pack2_bf16(x[4 * g + 2] * a.scale, x[4 * g + 3] * a.scale));
        *reinterpret_cast<uint2*>(a.dv + o) =
            make_uint2(pack2_bf16(y[4 * g], y[4 * g + 1]), pack2_bf16(y[4 * g + 2], y[4 * g + 3]));
      }
    }
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

template <int D, int NW, bool DENSE>
static hipError_t launch_passes(const BwdArgs& a, hipStream_t stream) {
  constexpr int ROWS = 32 * NW;
  const int64_t nq = (int64_t)a.bh * a.lq * D, nk = (int64_t)a.bh * a.lk * D;
  auto sum = [&](const float* part, int64_t stride, int ranges, int64_t n, float scale, uint16_t* out) {
    attn_bwd_sum_kernel<<<(n / 8 + 255) / 256, 256, 0, stream>>>(part, stride, ranges, n, scale, out);
  };
  const int64_t dq_grid = (int64_t)a.bh * a.dq_ranges * ((a.lq + ROWS - 1) / ROWS);
  if (dq_grid > 0) attn_bwd_dq_kernel<D, NW, DENSE><<<dq_grid, 64 * NW, 0, stream>>>(a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (a.dq_ranges > 1) sum(a.part, nq, a.dq_ranges, nq, a.scale, a.dq);
  const int64_t dkv_grid = (int64_t)a.bh * a.dkv_ranges * ((a.lk + ROWS - 1) / ROWS);
  attn_bwd_dkv_kernel<D, NW, DENSE><<<dkv_grid, 64 * NW, 0, stream>>>(a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (a.dkv_ranges > 1) {
    sum(a.part, 2 * nk, a.dkv_ranges, nk, a.scale, a.dk);
    sum(a.part + nk, 2 * nk, a.dkv_ranges, nk, 1.f, a.dv);
  }
  return hipGetLastError();
}

template <int D>
static hipError_t launch_bwd(const BwdArgs& a, bool dense, hipStream_t stream) {
  const int64_t rows = (int64_t)a.bh * a.n_q * a.block;
  constexpr int RPW = 256 / (D / 8);
  if (rows > 0) attn_bwd_stats_kernel<D><<<(rows + RPW - 1) / RPW, 256, 0, stream>>>(a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  if (dense) return launch_passes<D, 4, true>(a, stream);
  const dim3 grid((unsigned)((int64_t)a.bh * a.n_words), (unsigned)((a.n_k + kBitsChunk - 1) / kBitsChunk));
  if (rows > 0) attn_bwd_bits_kernel<<<grid, 1024, 0, stream>>>(a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  return a.block == 64 ? launch_passes<D, 2, false>(a, stream) : launch_passes<D, 4, false>(a, stream);
}

hipError_t launch_attn_bwd(const BwdArgs& a, int d, bool dense, hipStream_t stream) {
  return d == 128 ? launch_bwd<128>(a, dense, stream) : launch_bwd<64>(a, dense, stream);
}

}  // namespace sparstar
