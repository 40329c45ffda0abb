// Attention over the 8-bit key/value cache (cache.hip), dense or over block lists.
//
// K and V stay 8-bit codes in memory, L2 and on the way into LDS: a tile moves half the
// bytes of a bf16 one.  The roundings are those of the bf16 forward: P to bf16 once, O to
// bf16 once, and in between, where a list is cut into ranges, each range's sums to fp16
// (store_rows); all other sums are fp32.
//
// Two kernels.  Calls of more than 32 query rows are bound by the matrix cores and the
// VALU (cache_attn_kernel.h); up to 32 rows, single tokens above all, they stream the cache
// (cache_token_kernel).
#include "cache_attn_kernel.h"

namespace sparstar {

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

// ---- up to 32 query rows: one work-group of four waves per (head, range of the list); each
// wave has a share of the range, a ring of tiles of its own and no barrier until the four
// join what they found through LDS.  S^T = K Q^T and O^T += V^T P^T as in attn_fwd.hip, with
// the operands turned into bf16 in registers; mostly empty products, but the matrix cores
// could take 34 TB/s of codes this way.  A lone wave needs 0.7 us per tile, so what counts
// is how many there are: the call cuts its lists for four waves per CU.  24 heads of 144,512
// rows: 160 us, 5.6 TB/s of some 6.2 that reading reaches, with two tiles in LDS per wave (177
// with three or four); one head 24.5 us, and 30.2 with every wave's result joined through
// memory; 8 heads of 1,152 rows, D = 64, 10.7 us in one launch.
template <int D, bool DENSE>
__global__ __launch_bounds__(64 * kTokenWaves) __attribute__((amdgpu_waves_per_eu(2, 2)))
void cache_token_kernel(CacheAttnArgs a) {
  using C = CacheCfg<D>;
  constexpr int RING = 2, W = kTokenWaves;
  // a wave's K and V tiles, and then what it adds to the row's sums
  static_assert(2 * RING * C::TILE >= C::DT * 16 * 64 * 4, "a wave's sums fit its tiles");
  __shared__ __attribute__((aligned(1024))) uint8_t tiles[W][2][RING][C::TILE];
  __shared__ float meta[W][3][64];
  const int64_t bh = blockIdx.x / a.ranges;
  const int range = (int)(blockIdx.x - bh * a.ranges);
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int l32 = lane % 32, hh = lane / 32;
  auto& ks = tiles[wave][0];
  auto& vs = tiles[wave][1];

  // tokens that exist: rows past them are neither read nor attended to
  int64_t len = a.lk;
  if (a.lens != nullptr) {
    const int n = a.lens[bh / a.heads];
    len = n < 0 ? 0 : (n < a.lk ? n : a.lk);
  }
  const int n_blk = (int)((len + a.block - 1) / a.block);

  // Q as the B operand of S^T = K Q^T.  A 16-byte read of a K row feeds two k-steps, so
  // step 2 i + j covers columns 32 i + 16 h + 8 j + (0..7).
  const int64_t row = l32;
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
      const int64_t r = bh;  // (one query block)
      n = a.kv_num_blocks[r];
      n = n < 0 ? 0 : (n > a.stride ? a.stride : n);
      list = a.kv_indices + r * a.stride;
    }
    const int part = range * W + wave, parts = a.ranges * W;
    first = __builtin_amdgcn_readfirstlane((int)((int64_t)n * part / parts));
    cnt = __builtin_amdgcn_readfirstlane((int)((int64_t)n * (part + 1) / parts)) - first;
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

  uint32_t loff[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = C::RPD * i + lane / C::CPR;
    loff[i] = (uint32_t)(r * C::RB + 16 * ((lane % C::CPR) ^ cache_swz<D>(r)) - 1024 * i);
  }
  const uint8_t* const kbase = a.k_cache + bh * a.cap * D;
  const uint8_t* const vbase = a.v_cache + bh * a.cap * D;
  auto issue = [&](int tile, int slot) {
    int64_t left = tile < 0 ? 0 : len - (int64_t)tile * C::KB;
    left = left < 0 ? 0 : (left > C::KB ? C::KB : left);
    const int64_t at = tile < 0 ? 0 : (int64_t)tile * C::TILE;
    const uint32_t bytes = (uint32_t)left * C::RB;
    dma_tile<4>(__builtin_amdgcn_readfirstlane(lds_addr(ks[slot])), loff, raw_rsrc(kbase + at, bytes));
    dma_tile<4>(__builtin_amdgcn_readfirstlane(lds_addr(vs[slot])), loff, raw_rsrc(vbase + at, bytes));
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
    Tile ahead[RING - 1];
    ahead[0] = cur;
    issue(cur.t, 0);
#pragma unroll
    for (int i = 1; i < RING - 1; ++i) {
      ahead[i] = fetch(i);
      issue(ahead[i].t, i);
    }
    int slot = 0;
    for (int j = 0; j < ntiles; ++j) {
      const Tile nt = fetch(j + RING - 1);
      wait_loads_and_lds<2 * 4 * (RING - 2)>();  // tile j, with the tiles issued after it outstanding
      asm volatile("" ::: "memory");
      issue(nt.t, slot == 0 ? RING - 1 : slot - 1);
      cur = ahead[0];
#pragma unroll
      for (int i = 0; i + 1 < RING - 1; ++i) ahead[i] = ahead[i + 1];
      ahead[RING - 2] = nt;
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
      slot = slot + 1 == RING ? 0 : slot + 1;
    }
    wait_vmcnt<0>();  // loads past the end of the list still write LDS
    asm volatile("" ::: "memory");
  }

  // The first wave joins the four: with M = max_w m_w, sums of 2^(m_w - M) times each one's.
  float l = half_swap_sum(l_run), le = half_swap_sum(le_run);
  if (wave != 0) {
    float4* mine = reinterpret_cast<float4*>(&tiles[wave][0][0][0]) + lane;
#pragma unroll
    for (int i = 0; i < C::DT * 4; ++i) {
      const f32x16& x = acc[i / 4];
      mine[64 * i] = make_float4(x[4 * (i % 4)], x[4 * (i % 4) + 1], x[4 * (i % 4) + 2], x[4 * (i % 4) + 3]);
    }
    meta[wave][0][lane] = m_run;
    meta[wave][1][lane] = l;
    meta[wave][2][lane] = le;
  }
  __syncthreads();
  if (wave != 0) return;
  float m = m_run;
#pragma unroll
  for (int w = 1; w < W; ++w) m = fmaxf(m, meta[w][0][lane]);
  // (a wave that saw no key has m = -inf and sums of zero, a NaN among its sums passes on)
  auto weight = [&](float x) { return x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x - m); };
  const float own = weight(m_run);
  l *= own;
  le *= own;
#pragma unroll
  for (int t = 0; t < C::DT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[t][e] *= own;
#pragma unroll
  for (int w = 1; w < W; ++w) {
    const float f = weight(meta[w][0][lane]);
    l = fmaf(meta[w][1][lane], f, l);
    le = fmaf(meta[w][2][lane], f, le);
    const float4* theirs = reinterpret_cast<const float4*>(&tiles[w][0][0][0]) + lane;
#pragma unroll
    for (int i = 0; i < C::DT * 4; ++i) {
      const float4 u = theirs[64 * i];
      f32x16& x = acc[i / 4];
      const int e = 4 * (i % 4);
      x[e] = fmaf(u.x, f, x[e]), x[e + 1] = fmaf(u.y, f, x[e + 1]);
      x[e + 2] = fmaf(u.z, f, x[e + 2]), x[e + 3] = fmaf(u.w, f, x[e + 3]);
    }
  }
  store_rows<D, Codes8>(a, bh, row, range, acc, m, l, le, hh);
}

template <int D, bool DENSE>
static hipError_t launch_mode(const CacheAttnArgs& a, int waves, hipStream_t stream) {
  if (waves == 1) {
    cache_token_kernel<D, DENSE><<<(int64_t)a.bh * a.ranges, 64 * kTokenWaves, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    return launch_merge<D, 16, Codes8>(a, stream);
  }
  return launch_rows<D, DENSE, Codes8>(a, waves, cache_join_groups(waves, (int64_t)a.bh * a.lq, a.ranges), stream);
}

hipError_t launch_cache_attn(const CacheAttnArgs& a, int d, int waves, bool dense, hipStream_t stream) {
  if (d == 128) return dense ? launch_mode<128, true>(a, waves, stream) : launch_mode<128, false>(a, waves, stream);
  return dense ? launch_mode<64, true>(a, waves, stream) : launch_mode<64, false>(a, waves, stream);
}

}  // namespace sparstar
