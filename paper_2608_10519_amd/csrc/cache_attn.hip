// Attention over the 8-bit key/value cache (cache.hip), dense or over block lists.
//
// K and V stay 8-bit codes in memory, L2 and LDS: each tile moves half the bytes of a
// bf16 one.  A lane turns the operands that it feeds to the matrix cores into bf16 in
// registers, where code * 2^e is exact, so the only roundings are those of the bf16
// forward: P to bf16 once, O to bf16 once.
//
// One work-group per (head, range of the list, 32 NW queries), one wave per 32
// queries; S^T = K Q^T and O^T += V^T P^T as in attn_fwd.hip, whose MFMA layouts hold
// here too.
#include "attn_device.h"

namespace sparstar {

template <int D, int NW>
struct CacheCfg {
  static constexpr int KB = attn_tile_keys(D);    // keys per tile
  static constexpr int KT = KB / 32;              // 32-key sub-tiles
  static constexpr int DS = D / 16, DT = D / 32;  // MFMA k-steps over D, 32-row tiles of O^T
  static constexpr int RB = D;                    // bytes per row
  static constexpr int CPR = D / 16;              // 16-byte chunks per row
  static constexpr int RPD = 1024 / RB;           // rows per direct-to-LDS wave load
  static constexpr int TILE = KB * RB;            // bytes per tile: 4 KB
  static constexpr int N = 4 / NW;                // direct loads per wave and tile
  static constexpr int RING = NW == 1 ? 4 : 3;    // tiles held in LDS, K and V each
  static_assert(TILE == 4096, "4 KB tiles");
};

// The chunks of a row are XOR-permuted so that both reads of a tile are free of bank
// conflicts: 16 consecutive rows of one chunk (ds_read_b128), and rows 4 h + 0..3 and
// 8 + 4 h + 0..3 of two chunks (the 8-bit transpose read).
template <int D>
__device__ __forceinline__ int cache_swz(int r) {
  if (D == 128) {
    const int p = (r >> 1) & 7;  // two rows per pass over the banks
    return (p & 4) | (p & 1) << 1 | (p >> 1 & 1);
  }
  return (r >> 2) & 3;  // four
}

// eight codes -> eight bf16 values times the scale (exact)
__device__ __forceinline__ bf16x8 decode8(uint2 u, float scale) {
  uint4 r;
  r.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.x, scale, false));
  r.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.x, scale, true));
  r.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.y, scale, false));
  r.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u.y, scale, true));
  return __builtin_bit_cast(bf16x8, r);
}

typedef int i32x2 __attribute__((ext_vector_type(2)));
// The 8-bit transpose read: in each 16-lane group, source lanes 2 k and 2 k + 1 point at
// the two halves of row k's 16 bytes, and lane j receives byte j of rows 0..7.
__device__ __forceinline__ uint2 lds_read_tr8(const uint8_t* p) {
  const i32x2 r = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
      (__attribute__((address_space(3))) i32x2*)(const_cast<uint8_t*>(p)));
  return make_uint2((uint32_t)r[0], (uint32_t)r[1]);
}

// At most n vector loads outstanding, and no LDS read: a single wave has no barrier that
// would order its reads of a tile before the loads that overwrite it.
template <int N>
__device__ __forceinline__ void wait_loads_and_lds() {
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
}

template <int D, int NW, bool DENSE>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2)))
void cache_attn_kernel(CacheAttnArgs a) {
  using C = CacheCfg<D, NW>;
  constexpr int ROWS = 32 * NW;
  __shared__ __attribute__((aligned(1024))) uint8_t ks[C::RING][C::TILE];
  __shared__ __attribute__((aligned(1024))) uint8_t vs[C::RING][C::TILE];
  const int64_t n_g = (a.lq + ROWS - 1) / ROWS;
  const int64_t w = xcd_linear(blockIdx.x, gridDim.x);
  const int64_t pair = w / n_g;
  const int qg = (int)(w - pair * n_g);
  const int64_t bh = pair / a.ranges;
  const int range = (int)(pair - bh * a.ranges);
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int l32 = lane % 32, hh = lane / 32;

  // tokens that exist: rows past them are neither read nor attended to
  int64_t len = a.lk;
  if (a.lens != nullptr) {
    const int n = a.lens[bh / a.heads];
    len = n < 0 ? 0 : (n < a.lk ? n : a.lk);
  }
  const int n_blk = (int)((len + a.block - 1) / a.block);

  // Q as the B operand of S^T = K Q^T.  A 16-byte read of a K row feeds two k-steps, so
  // step 2 i + j covers columns 32 i + 16 h + 8 j + (0..7).
  const int64_t row = (int64_t)qg * ROWS + wave * 32 + l32;
  const bool row_ok = row < a.lq;
  bf16x8 qf[C::DS];
#pragma unroll
  for (int s = 0; s < C::DS; ++s) {
    const uint16_t* p = a.q + (bh * a.lq + (row_ok ? row : 0)) * D + 32 * (s / 2) + 16 * hh + 8 * (s % 2);
    const uint4 u = row_ok ? *reinterpret_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0);
    qf[s] = __builtin_bit_cast(bf16x8, u);
  }

  // The range's key blocks: an even share of the list's entries, or of all blocks.
  int first = 0, cnt;
  const int32_t* list = nullptr;
  {
    int n = n_blk;
    if constexpr (!DENSE) {
      const int64_t r = bh * a.n_q + (int64_t)qg * ROWS / a.block;
      n = a.kv_num_blocks[r];
      n = n < 0 ? 0 : (n > a.stride ? a.stride : n);
      list = a.kv_indices + r * a.stride;
    }
    first = __builtin_amdgcn_readfirstlane((int)((int64_t)n * range / a.ranges));
    cnt = __builtin_amdgcn_readfirstlane((int)((int64_t)n * (range + 1) / a.ranges)) - first;
  }
  // Entries 64 at a time in VGPRs: the block and its scale bytes.  One that names no
  // block gives -1, whose tiles are loaded as zeros and masked.
  const int sub_bits = __builtin_ctz(a.block / C::KB);
  const int64_t scale_at = bh * ((a.cap + a.block - 1) / a.block);
  int breg = -1, sreg = 0, lbase = 0;
  auto load_batch = [&](int base) {
    lbase = base;
    int b = -1;
    if (base + lane < cnt) b = DENSE ? first + base + lane : list[first + base + lane];
    if (b >= n_blk || b < 0) b = -1;
    breg = b;
    sreg = 127 | 127 << 8;
    if (b >= 0) sreg = (int)a.k_scale[scale_at + b] | (int)a.v_scale[scale_at + b] << 8;
    asm volatile("; list batch %0 %1" ::"v"(breg), "v"(sreg));
  };
  const int ntiles = cnt << sub_bits;
  struct Tile {
    int t;     // KB-key tile of the cache, -1: none
    int s;     // scale bytes
  };
  auto fetch = [&](int j) -> Tile {
    const int e = j >> sub_bits;
    if (j >= ntiles) return Tile{-1, 127 | 127 << 8};
    if (e >= lbase + 64) load_batch(lbase + 64);
    const int b = __builtin_amdgcn_readlane(breg, e - lbase), s = __builtin_amdgcn_readlane(sreg, e - lbase);
    return Tile{b < 0 ? -1 : (b << sub_bits) + (j & ((1 << sub_bits) - 1)), s};
  };

  uint32_t loff[C::N];
#pragma unroll
  for (int i = 0; i < C::N; ++i) {
    const int r = C::RPD * (C::N * wave + i) + lane / C::CPR;
    loff[i] = (uint32_t)(r * C::RB + 16 * ((lane % C::CPR) ^ cache_swz<D>(r)) - 1024 * i);
  }
  const uint8_t* const kbase = a.k_cache + bh * a.cap * D;
  const uint8_t* const vbase = a.v_cache + bh * a.cap * D;
  auto issue = [&](int tile, int slot) {
    int64_t left = tile < 0 ? 0 : len - (int64_t)tile * C::KB;
    left = left < 0 ? 0 : (left > C::KB ? C::KB : left);
    const int64_t at = tile < 0 ? 0 : (int64_t)tile * C::TILE;
    const uint32_t bytes = (uint32_t)left * C::RB, m0 = (uint32_t)(C::N * wave) * 1024u;
    dma_tile<C::N>(lds_addr(ks[slot]) + m0, loff, raw_rsrc(kbase + at, bytes));
    dma_tile<C::N>(lds_addr(vs[slot]) + m0, loff, raw_rsrc(vbase + at, bytes));
  };

  // per-lane LDS offsets: K row l32, chunk 2 i + h; V rows of the transpose read
  uint32_t koff[C::DS / 2], voff[C::DT];
#pragma unroll
  for (int i = 0; i < C::DS / 2; ++i) koff[i] = (uint32_t)(l32 * C::RB + 16 * ((2 * i + hh) ^ cache_swz<D>(l32)));
  {
    const int k = (lane & 15) >> 1, r = 4 * hh + (k & 3) + (k >= 4 ? 8 : 0);
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
      voff[t] = (uint32_t)(r * C::RB + 16 * ((2 * t + (lane >> 4 & 1)) ^ cache_swz<D>(r)) + 8 * (lane & 1));
  }

  f32x16 acc[C::DT];
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] = 0.f;
  float m_run = -INFINITY, l_run = 0.f, le_run = 0.f;  // max in the log2 domain; sums of the lane's half of the keys

  if (ntiles > 0) {
    load_batch(0);
    Tile cur = fetch(0);
    Tile ahead[C::RING - 1];
    ahead[0] = cur;
    issue(cur.t, 0);
#pragma unroll
    for (int i = 1; i < C::RING - 1; ++i) {
      ahead[i] = fetch(i);
      issue(ahead[i].t, i);
    }
    int slot = 0;
    for (int j = 0; j < ntiles; ++j) {
      const Tile nt = fetch(j + C::RING - 1);
      wait_loads_and_lds<2 * C::N*(C::RING - 2)>();  // tile j, with the tiles issued after it outstanding
      __syncthreads();
      issue(nt.t, slot == 0 ? C::RING - 1 : slot - 1);
      cur = ahead[0];
#pragma unroll
      for (int i = 0; i + 1 < C::RING - 1; ++i) ahead[i] = ahead[i + 1];
      ahead[C::RING - 2] = nt;
      const uint8_t* kt_lds = ks[slot];
      const uint8_t* vt_lds = vs[slot];
      const float ksc = __uint_as_float((uint32_t)(cur.s & 255) << 23);
      const float vsc = __uint_as_float((uint32_t)(cur.s >> 8) << 23);
      f32x16 s[C::KT];
      float mx = -INFINITY;
      const int64_t left = cur.t < 0 ? 0 : len - (int64_t)cur.t * C::KB;
#pragma unroll
      for (int kt = 0; kt < C::KT; ++kt) {
#pragma unroll
        for (int e = 0; e < 16; ++e) s[kt][e] = 0.f;
#pragma unroll
        for (int i = 0; i < C::DS / 2; ++i) {
          const uint4 u = *reinterpret_cast<const uint4*>(kt_lds + koff[i] + kt * 32 * C::RB);
          s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode8(make_uint2(u.x, u.y), ksc), qf[2 * i], s[kt], 0, 0, 0);
          s[kt] =
              __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode8(make_uint2(u.z, u.w), ksc), qf[2 * i + 1], s[kt], 0, 0, 0);
        }
        if (left < C::KB) {
          const int vis = (int)(left < 0 ? 0 : left) - 32 * kt - 4 * hh;
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (8 * (e / 4) + e % 4 >= vis) s[kt][e] = -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[kt][e]);
      }
      mx = half_swap_max(mx) * a.scale_log2;
      if (__builtin_amdgcn_ballot_w64(mx > m_run)) {
        const float m_new = fmaxf(m_run, mx);
        const float alpha = m_new == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
        l_run *= alpha;
        le_run *= alpha;
#pragma unroll
        for (int t = 0; t < C::DT; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[t][e] *= alpha;
      }
      const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
#pragma unroll
      for (int kt = 0; kt < C::KT; ++kt) {
        u32x8 pk;
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(s[kt][e], a.scale_log2, neg_m));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(s[kt][e + 1], a.scale_log2, neg_m));
          const uint32_t u = pack2_bf16(p0, p1);
          le_run += p0 + p1;
          l_run += bf16_lo(u) + bf16_hi(u);
          pk[e / 2] = u;
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int t = 0; t < C::DT; ++t) {
            const uint2 u = lds_read_tr8(vt_lds + voff[t] + (32 * kt + 16 * half) * C::RB);
            acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(decode8(u, vsc), pack_half(pk, half), acc[t], 0, 0, 0);
          }
      }
      slot = slot + 1 == C::RING ? 0 : slot + 1;
    }
    wait_vmcnt<0>();  // loads past the end of the list still write LDS
  }

  l_run = half_swap_sum(l_run);
  le_run = half_swap_sum(le_run);
  if (!row_ok) return;
  const int64_t at = bh * a.lq + row;
  if (a.ranges > 1) {
    const int64_t prow = (int64_t)range * a.bh * a.lq + at;
    float* out = a.part_o + prow * D + 4 * hh;
#pragma unroll
    for (int t = 0; t < C::DT; ++t)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(out + 32 * t + 8 * g) =
            make_float4(acc[t][4 * g], acc[t][4 * g + 1], acc[t][4 * g + 2], acc[t][4 * g + 3]);
    if (hh == 0) reinterpret_cast<float4*>(a.part_meta)[prow] = make_float4(m_run, l_run, le_run, 0.f);
    return;
  }
  const float inv = l_run == 0.f ? 0.f : 1.f / l_run;  // (a NaN passes on)
  uint16_t* out = a.o + at * D + 4 * hh;
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<uint2*>(out + 32 * t + 8 * g) =
          make_uint2(pack2_bf16(acc[t][4 * g] * inv, acc[t][4 * g + 1] * inv),
                     pack2_bf16(acc[t][4 * g + 2] * inv, acc[t][4 * g + 3] * inv));
  if (a.lse != nullptr && hh == 0)
    a.lse[at] = le_run == 0.f ? -INFINITY : (m_run + log2f(le_run)) * 0.69314718055994530942f;
}

// Joins the ranges of one row: with M = max_r m_r and w_r = 2^(m_r - M),
// O = sum w_r A_r / sum w_r l_r and lse = ln 2 (M + log2 sum w_r le_r).  D / 8 threads
// per row and G groups of them, each over every G-th range.
template <int D, int G>
__global__ __launch_bounds__(256) void cache_merge_kernel(CacheAttnArgs a) {
  constexpr int LPR = D / 8, RPB = 256 / (LPR * G);
  __shared__ float red[G][RPB][LPR][8];
  const int c = threadIdx.x % LPR, g = threadIdx.x / LPR % G, rb = threadIdx.x / (LPR * G);
  const int64_t rows = (int64_t)a.bh * a.lq, row = (int64_t)blockIdx.x * RPB + rb;
  const bool ok = row < rows;
  float m = -INFINITY, l = 0.f, le = 0.f;
  const float4* meta = reinterpret_cast<const float4*>(a.part_meta);
  if (ok)
    for (int r = 0; r < a.ranges; ++r) {
      const float4 x = meta[(int64_t)r * rows + row];
      const float mn = fmaxf(m, x.x);
      if (x.y != 0.f) {
        const float s = __builtin_amdgcn_exp2f(m - mn), t = __builtin_amdgcn_exp2f(x.x - mn);
        l = l * s + x.y * t;
        le = le * s + x.z * t;
        m = mn;
      }
    }
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (ok)
    for (int r = g; r < a.ranges; r += G) {
      const int64_t p = (int64_t)r * rows + row;
      const float4 x = meta[p];
      const float4 u = *reinterpret_cast<const float4*>(a.part_o + p * D + 8 * c);
      const float4 v = *reinterpret_cast<const float4*>(a.part_o + p * D + 8 * c + 4);
      if (x.y == 0.f) continue;  // no key seen; NaN passes on
      const float t = __builtin_amdgcn_exp2f(x.x - m);
      acc[0] = fmaf(t, u.x, acc[0]), acc[1] = fmaf(t, u.y, acc[1]);
      acc[2] = fmaf(t, u.z, acc[2]), acc[3] = fmaf(t, u.w, acc[3]);
      acc[4] = fmaf(t, v.x, acc[4]), acc[5] = fmaf(t, v.y, acc[5]);
      acc[6] = fmaf(t, v.z, acc[6]), acc[7] = fmaf(t, v.w, acc[7]);
    }
  if constexpr (G > 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) red[g][rb][c][e] = acc[e];
    __syncthreads();
    if (g != 0) return;
#pragma unroll
    for (int i = 1; i < G; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += red[i][rb][c][e];
  }
  if (!ok) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<uint4*>(a.o + row * D + 8 * c) =
      make_uint4(pack2_bf16(acc[0] * inv, acc[1] * inv), pack2_bf16(acc[2] * inv, acc[3] * inv),
                 pack2_bf16(acc[4] * inv, acc[5] * inv), pack2_bf16(acc[6] * inv, acc[7] * inv));
  if (a.lse != nullptr && c == 0) a.lse[row] = le == 0.f ? -INFINITY : (m + log2f(le)) * 0.69314718055994530942f;
}

template <int D, int NW, bool DENSE>
static hipError_t launch_rows(const CacheAttnArgs& a, hipStream_t stream) {
  const int64_t grid = (int64_t)a.bh * a.ranges * ((a.lq + 32 * NW - 1) / (32 * NW));
  cache_attn_kernel<D, NW, DENSE><<<grid, 64 * NW, 0, stream>>>(a);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || a.ranges == 1) return e;
  const int64_t rows = (int64_t)a.bh * a.lq;
  if (NW == 1) {
    constexpr int RPB = 256 / (D / 8 * 16);
    cache_merge_kernel<D, 16><<<(rows + RPB - 1) / RPB, 256, 0, stream>>>(a);
  } else {
    constexpr int RPB = 256 / (D / 8);
    cache_merge_kernel<D, 1><<<(rows + RPB - 1) / RPB, 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

template <int D>
static hipError_t launch_d(const CacheAttnArgs& a, int waves, bool dense, hipStream_t stream) {
  if (waves == 1) return dense ? launch_rows<D, 1, true>(a, stream) : launch_rows<D, 1, false>(a, stream);
  if (waves == 2) return dense ? launch_rows<D, 2, true>(a, stream) : launch_rows<D, 2, false>(a, stream);
  return dense ? launch_rows<D, 4, true>(a, stream) : launch_rows<D, 4, false>(a, stream);
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, int d, int waves, bool dense, hipStream_t stream) {
  return d == 128 ? launch_d<128>(a, waves, dense, stream) : launch_d<64>(a, waves, dense, stream);
}

}  // namespace sparstar
