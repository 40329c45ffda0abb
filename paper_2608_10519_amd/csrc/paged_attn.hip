// Attention over the paged 4-bit key/value cache (paged.hip), dense or over block lists.
#include "cache_attn_kernel.h"

namespace sparstar {

// Cache policy of the codes' loads, nt: each is read once a call.  20 x 24 heads of 20,000 rows
// 207 us, 232 with the plain policy.
constexpr int kOnce = 2;

__device__ __forceinline__ uint32_t scale_byte(__amdgpu_buffer_rsrc_t rs, int at) {
  return __builtin_amdgcn_raw_buffer_load_b8(rs, at, 0, 0);
}

// ---- up to 32 query rows: one work-group of W waves per (head, range of the list); each wave
// has a share of the range's 64-key tiles and no barrier until the waves join what they found.
//
// A long cache is read once, at what memory gives: one row of 24 heads, D = 128, 144,512 rows
// 77 us, 6.1 TB/s; 20 x 24 heads of 20,000 rows 205 us, 6.4 TB/s; 32 rows of the first 97 us; D = 64
// 45 us.  A short one is bound by the wave that walks its tiles one after the other, 1.1 us each
// at D = 128 and 0.7 at D = 64 where the wave is alone on its SIMD (loads, conversions, two
// products and a softmax that wait for each other): 8 heads of 1,152 rows, D = 64, 7.5 us.  So
// everything stays in the wave: with 32 x 32 products half of them would be padding, and K in LDS
// would be one more step that waits.
//
// On v_mfma_f32_16x16x32_bf16 (lane l, j = l / 16: A[m][k] m = l % 16, B[k][n] n = l % 16, k =
// 8 j + i of the lane's eight; C[m][n] n = l % 16, m = 4 j + a):
//   * S^T = K Q^T, 16 keys a product.  A lane loads the D / 4 channels G j .. of key l % 16
//     straight into registers (16 rows: 1 KB in a row) and decodes them eight at a time; Q's
//     operand takes the same order of channels;
//   * softmax in the log2 domain against a running max that is only refreshed when some
//     lane's sum of a tile's P exceeds 2^8;
//   * O^T += V^T P^T, 32 keys a product: P is in S's layout, keys 16 (i / 4) + 4 j + i % 4, and
//     V's operand comes in that order from LDS: a lane loads 32 channels of a key, decodes
//     them and stores them as bf16 rows, which the transpose read takes by columns.  A product
//     with ones sums the rounded P.
// P is rounded to bf16 because the products take both operands in one type and V has no other
// of 16 bits: its scales reach far past fp16's range.  A weight is off by at most 2^-8 of itself,
// O by about as much as by its own rounding to bf16 (0.0017 of it, 0.0024 with both); P as a sum
// of two bf16 numbers would double the products of P V.
template <int D, int NC, bool DENSE, int W>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(2, 2)))
void paged_token_kernel(PagedAttnArgs a) {
  // tiles whose loads are in flight: 32 rows at D = 128 have no registers for two
  constexpr int AHEAD = D * NC > 128 ? 1 : 2;
  constexpr int KS = D / 32;           // k-steps of S
  constexpr int DT = D / 16;           // 16-channel tiles of O^T
  constexpr int KW = D / 32;           // dwords of K codes per lane and 16 keys
  constexpr int LPK = D / 32;          // lanes per key of a V load
  constexpr int VL = LPK;              // V loads per tile: 64 / LPK keys each
  constexpr int RB = 2 * D;            // bytes of a bf16 row
  constexpr int VT = 64 * RB;
  static_assert(VT >= DT * NC * 64 * 16, "a wave's sums fit its tile");
  __shared__ __attribute__((aligned(1024))) uint8_t tiles[W][VT];
  __shared__ float meta[W][3][16 * NC];
  const uint32_t head = blockIdx.x / (uint32_t)a.ranges;
  const int range = (int)(blockIdx.x - head * (uint32_t)a.ranges);
  const int64_t bh = head, b = head / (uint32_t)a.heads, h = head % (uint32_t)a.heads;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int l16 = lane % 16, j = lane / 16;

  // (both counts are loaded before either is waited for)
  int given = 0, listed = 0;
  if (a.lens != nullptr) given = a.lens[b];
  if constexpr (!DENSE) listed = a.kv_num_blocks[bh];  // (one query block)
  const int64_t len = a.lens == nullptr ? a.lk : (given < 0 ? 0 : (given < a.lk ? given : a.lk));
  const int sub_bits = a.block == 128 ? 1 : 0;
  const int n_blk = (int)((len + a.block - 1) >> (6 + sub_bits));

  // Q[n][(D / 4) j + 8 s + i]
  bf16x8 qf[NC][KS];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int64_t row = 16 * c + l16;
      uint4 u = make_uint4(0, 0, 0, 0);
      if (row < a.lq) u = *reinterpret_cast<const uint4*>(a.q + (bh * a.lq + row) * D + D / 4 * j + 8 * s);
      qf[c][s] = __builtin_bit_cast(bf16x8, u);
    }

  // The wave's 64-key tiles [first, end) of the list's (of all) blocks.
  int first, end;
  const int32_t* list = nullptr;
  {
    int n = n_blk;
    if constexpr (!DENSE) {
      n = listed < 0 ? 0 : (listed > a.stride ? a.stride : listed);
      list = a.kv_indices + bh * a.stride;
    }
    const uint32_t part = range * W + wave, parts = a.ranges * W, all = (uint32_t)n << sub_bits;
    const uint32_t each = all / parts, more = all - each * parts;  // the first `more` parts take one more
    first = __builtin_amdgcn_readfirstlane((int)(part * each + (part < more ? part : more)));
    end = first + (int)each + (part < more ? 1 : 0);
  }
  // Entries 64 at a time in VGPRs: the block and its page; -1 where there is none.
  int breg = -1, preg = 0, lbase = 0;
  auto load_batch = [&](int base) {
    lbase = base;
    int e = -1;
    if ((base + lane) << sub_bits < end) e = DENSE ? base + lane : list[base + lane];
    if (e < 0 || e >= n_blk) e = -1;
    preg = e < 0 ? -1 : a.pages[b * a.n_table + e];
    if (preg < 0 || preg >= a.n_pages) e = -1, preg = 0;
    breg = e;
    asm volatile("; list batch %0 %1" ::"v"(breg), "v"(preg));
  };
  struct Tile {
    int left;     // keys, <= 0: none
    int64_t row;  // of the pool
  };
  auto fetch = [&](int i) -> Tile {
    if (i >= end) return Tile{0, 0};
    const int e = i >> sub_bits, sub = i & ((1 << sub_bits) - 1);
    if (e >= lbase + 64) load_batch(lbase + 64);
    const int blk = __builtin_amdgcn_readlane(breg, e - lbase), page = __builtin_amdgcn_readlane(preg, e - lbase);
    const int64_t left = blk < 0 ? 0 : len - ((int64_t)blk * a.block + 64 * sub);
    return Tile{(int)(left < 0 ? 0 : (left > 64 ? 64 : left)), ((int64_t)page * a.heads + h) * a.block + 64 * sub};
  };

  struct Raw {
    uint32_t k[4][KW], ks[4];  // by 16 keys
    uint4 v[VL];
    uint32_t vs[VL];
  };
  const int kat = l16 * (D / 2) + j * (D / 8), ksat = l16 * (D / 32) + j * (D / 32) / 4;
  auto load = [&](Tile t, Raw& r) {
    const uint32_t n = (uint32_t)t.left;
    const auto kr = tile_rsrc(a.k_cache + t.row * (D / 2), n * (D / 2)), vr = tile_rsrc(a.v_cache + t.row * (D / 2), n * (D / 2));
    const auto ksr = tile_rsrc(a.k_scale + t.row * (D / 32), n * (D / 32));
    const auto vsr = tile_rsrc(a.v_scale + t.row * (D / 32), n * (D / 32));
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if constexpr (D == 128) {
        const uint4 w = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(kr, kat + 1024 * u, 0, kOnce));
        r.k[u][0] = w.x, r.k[u][1] = w.y, r.k[u][2] = w.z, r.k[u][3] = w.w;
      } else {
        const uint2 w = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(kr, kat + 512 * u, 0, kOnce));
        r.k[u][0] = w.x, r.k[u][1] = w.y;
      }
      r.ks[u] = scale_byte(ksr, ksat + 16 * (D / 32) * u);
    }
#pragma unroll
    for (int u = 0; u < VL; ++u) {
      r.v[u] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(vr, 16 * lane + 1024 * u, 0, kOnce));
      r.vs[u] = scale_byte(vsr, lane + 64 * u);
    }
  };

  // V in LDS: the chunks of row r are permuted so that eight consecutive rows' pairs of chunks
  // (the transpose read, 256 bytes of banks) and what eight lanes store (chunks four apart of two
  // rows, or of four at D = 64, 128 bytes of banks) fall on different ones.
  auto swz = [](int r, int c) { return D == 128 ? 2 * (r & 7) ^ c >> 3 : 2 * ((r >> 1) & 3) ^ (r & 1); };
  uint8_t* const vt = tiles[wave];
  const int vrow = lane / LPK, vc = 4 * (lane % LPK);
  uint32_t vput[4], vget[DT];
#pragma unroll
  for (int i = 0; i < 4; ++i) vput[i] = (uint32_t)(vrow * RB + 16 * ((vc + i) ^ swz(vrow, vc + i)));
  {
    const int r = 4 * j + (lane & 15) / 4, p = lane & 3;  // rows 4 j .. + 3, four pieces of 8 bytes
#pragma unroll
    for (int t = 0; t < DT; ++t) vget[t] = (uint32_t)(r * RB + 16 * ((2 * t + p / 2) ^ swz(r, 2 * t + p / 2)) + 8 * (p % 2));
  }
  auto read_v = [&](int t, int half) -> bf16x8 {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(vt + vget[t] + 32 * half * RB);
    const s16x4 lo = lds_read_tr(p), hi = lds_read_tr(p + 16 * D);
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };

  f32x4 acc[DT][NC], accl[NC];
  float m_run[NC], le_run[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    accl[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[c] = -INFINITY, le_run[c] = 0.f;
  }
  const uint32_t one2 = 0x3f803f80u;
  const bf16x8 ones = __builtin_bit_cast(bf16x8, make_uint4(one2, one2, one2, one2));

  auto step = [&](Tile cur, const Raw& r) {
    f32x4 s[4][NC];
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int c = 0; c < NC; ++c) s[u][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < 4 * KS; ++n) {
      // the four sums in turn, so that a product waits for none of its neighbours (two columns
      // are two sums already, and have no registers for more)
      const int u = NC == 1 ? n % 4 : n / KS, k = NC == 1 ? n / 4 : n % KS;
      const bf16x8 kv = decode8_4bit(r.k[u][k], __uint_as_float(r.ks[u] << 23));
#pragma unroll
      for (int c = 0; c < NC; ++c) s[u][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kv, qf[c][k], s[u][c], 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < VL; ++u) {
      const float sc = __uint_as_float(r.vs[u] << 23);
      const uint32_t w[4] = {r.v[u].x, r.v[u].y, r.v[u].z, r.v[u].w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<bf16x8*>(vt + vput[i] + u * (64 / LPK) * RB) = decode8_4bit(w[i], sc);
    }
    if (cur.left < 64) {
      asm volatile("; mask");
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (16 * u + 4 * j + e >= cur.left)
#pragma unroll
            for (int c = 0; c < NC; ++c) s[u][c][e] = -INFINITY;
    }
    bf16x8 pk[2][NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float p[16], se = 0.f;
      const float neg_m = m_run[c] == -INFINITY ? INFINITY : -m_run[c];  // (no key seen yet: takes the exact path)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        p[e] = __builtin_amdgcn_exp2f(fmaf(s[e / 4][c][e % 4], a.scale_log2, neg_m));
        se += p[e];
      }
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(!(se <= 256.f)) != 0, 0)) {
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e / 4][c][e % 4]);
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32)) * a.scale_log2;
        const float mn = fmaxf(m_run[c], mx), alpha = mn == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m_run[c] - mn);
        m_run[c] = mn;
        le_run[c] *= alpha;
#pragma unroll
        for (int e = 0; e < 4; ++e) accl[c][e] *= alpha;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[t][c][e] *= alpha;
        const float off = mn == -INFINITY ? 0.f : -mn;
        se = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(s[e / 4][c][e % 4], a.scale_log2, off));
          se += p[e];
        }
      }
      le_run[c] += se;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const float* x = p + 8 * half;
        pk[half][c] = __builtin_bit_cast(
            bf16x8, make_uint4(pack2_bf16(x[0], x[1]), pack2_bf16(x[2], x[3]), pack2_bf16(x[4], x[5]), pack2_bf16(x[6], x[7])));
      }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int c = 0; c < NC; ++c) accl[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pk[half][c], accl[c], 0, 0, 0);
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const bf16x8 v = read_v(t, half);
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pk[half][c], acc[t][c], 0, 0, 0);
      }
    }
  };

  if (first < end) {
    load_batch(first >> sub_bits);
    // (A tile's loads stay in the order of the tiles, which is that of the waits.)
    auto next = [&](int i, Tile& t, Raw& r) {
      __builtin_amdgcn_sched_barrier(0);
      t = fetch(i);
      load(t, r);
      __builtin_amdgcn_sched_barrier(0);
    };
    Tile t0, t1;
    Raw r0, r1;
    next(first, t0, r0);
    if constexpr (AHEAD == 1) {
      for (int i = first; i < end; ++i) {
        step(t0, r0);
        next(i + 1, t0, r0);
      }
    } else {
      next(first + 1, t1, r1);
      int i = first;
      for (; i + 1 < end; i += 2) {  // (no way out in between, which would make every wait one for all loads)
        step(t0, r0);
        next(i + 2, t0, r0);
        step(t1, r1);
        next(i + 3, t1, r1);
      }
      if (i < end) step(t0, r0);
    }
  }

  // The waves join: with M = max_w m_w, sums of 2^(m_w - M) times each one's, every wave for some
  // of the tiles of O^T.
  float4* const mine = reinterpret_cast<float4*>(vt) + lane;
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int c = 0; c < NC; ++c) mine[64 * (t * NC + c)] = make_float4(acc[t][c][0], acc[t][c][1], acc[t][c][2], acc[t][c][3]);
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float le = le_run[c];
    le += __shfl_xor(le, 16);
    le += __shfl_xor(le, 32);
    if (j == 0) meta[wave][0][16 * c + l16] = m_run[c], meta[wave][1][16 * c + l16] = accl[c][0], meta[wave][2][16 * c + l16] = le;
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int64_t row = 16 * c + l16;
    float m = -INFINITY, l = 0.f, le = 0.f, f[W];
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, meta[w][0][16 * c + l16]);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      // (a wave that saw no key has m = -inf and sums of zero, a NaN among its sums passes on)
      const float x = meta[w][0][16 * c + l16];
      f[w] = x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x - m);
      l = fmaf(meta[w][1][16 * c + l16], f[w], l);
      le = fmaf(meta[w][2][16 * c + l16], f[w], le);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t at = bh * a.lq + row, prow = (int64_t)range * a.bh * a.lq + at;
    if (wave == 0 && j == 0 && row < a.lq) {
      if (a.ranges > 1) reinterpret_cast<float4*>(a.part_meta)[prow] = make_float4(m, l, le, 0.f);
      else if (a.lse != nullptr) a.lse[at] = le == 0.f ? -INFINITY : (m + log2f(le)) * 0.69314718055994530942f;
    }
#pragma unroll
    for (int t = wave; t < DT; t += W) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float4 u = reinterpret_cast<const float4*>(tiles[w])[64 * (t * NC + c) + lane];
        x.x = fmaf(u.x, f[w], x.x), x.y = fmaf(u.y, f[w], x.y), x.z = fmaf(u.z, f[w], x.z), x.w = fmaf(u.w, f[w], x.w);
      }
      if (row >= a.lq) continue;
      if (a.ranges > 1) {
        *reinterpret_cast<float4*>(a.part32 + prow * D + 16 * t + 4 * j) = x;
      } else {
        *reinterpret_cast<uint2*>(a.o + at * D + 16 * t + 4 * j) =
            make_uint2(pack2_bf16(x.x * inv, x.y * inv), pack2_bf16(x.z * inv, x.w * inv));
      }
    }
  }
}

// Joins the ranges of a row, D / 4 threads and G groups of them, each over every G-th range: with
// 16 a thread reads four at most, all at once (64 ranges of one row 8.7 us with four groups).
constexpr int kJoinGroups = 16;
template <int D, int G>
__global__ __launch_bounds__(D / 4 * G) void paged_join_kernel(PagedAttnArgs a) {
  constexpr int LPR = D / 4;
  __shared__ float4 red[G][LPR];
  __shared__ float meta[G][3];
  const int c = threadIdx.x % LPR, g = threadIdx.x / LPR;
  const int64_t rows = (int64_t)a.bh * a.lq, row = blockIdx.x;
  float m = -INFINITY, l = 0.f, le = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  // (kPagedMaxRanges are four a thread: all loads at once)
  for (int r0 = 0; r0 < a.ranges; r0 += 4 * G) {
    float4 y[4], u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[i] = u[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r0 + i * G >= a.ranges) continue;
      const int64_t p = (int64_t)min(r0 + i * G + g, a.ranges - 1) * rows + row;
      y[i] = reinterpret_cast<const float4*>(a.part_meta)[p];
      u[i] = *reinterpret_cast<const float4*>(a.part32 + p * D + 4 * c);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (r0 + i * G + g >= a.ranges || y[i].y == 0.f) continue;  // no key seen; NaN passes on
      const float mn = fmaxf(m, y[i].x), s = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      const float t = y[i].x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(y[i].x - mn);
      l = fmaf(l, s, y[i].y * t), le = fmaf(le, s, y[i].z * t);
      x.x = fmaf(u[i].x, t, x.x * s), x.y = fmaf(u[i].y, t, x.y * s);
      x.z = fmaf(u[i].z, t, x.z * s), x.w = fmaf(u[i].w, t, x.w * s);
      m = mn;
    }
  }
  red[g][c] = x;
  if (c == 0) meta[g][0] = m, meta[g][1] = l, meta[g][2] = le;
  __syncthreads();
  if (g != 0) return;
  float mm = m;
#pragma unroll
  for (int i = 1; i < G; ++i) mm = fmaxf(mm, meta[i][0]);
  // (a group without keys has m = -inf and sums of zero, or NaN, which passes on)
  auto weight = [&](float v) { return v == -INFINITY ? (mm == -INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f(v - mm); };
  float s = weight(m);
  l *= s, le *= s, x.x *= s, x.y *= s, x.z *= s, x.w *= s;
#pragma unroll
  for (int i = 1; i < G; ++i) {
    s = weight(meta[i][0]);
    const float4 u = red[i][c];
    l = fmaf(meta[i][1], s, l), le = fmaf(meta[i][2], s, le);
    x.x = fmaf(u.x, s, x.x), x.y = fmaf(u.y, s, x.y), x.z = fmaf(u.z, s, x.z), x.w = fmaf(u.w, s, x.w);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *reinterpret_cast<uint2*>(a.o + row * D + 4 * c) =
      make_uint2(pack2_bf16(x.x * inv, x.y * inv), pack2_bf16(x.z * inv, x.w * inv));
  if (a.lse != nullptr && c == 0) a.lse[row] = le == 0.f ? -INFINITY : (mm + log2f(le)) * 0.69314718055994530942f;
}

template <int D, bool DENSE, int W>
static hipError_t launch_token(const PagedAttnArgs& a, hipStream_t stream) {
  const int64_t groups = (int64_t)a.bh * a.ranges;
  if (a.lq <= 16) paged_token_kernel<D, 1, DENSE, W><<<groups, 64 * W, 0, stream>>>(a);
  else paged_token_kernel<D, 2, DENSE, W><<<groups, 64 * W, 0, stream>>>(a);
  return hipGetLastError();
}

template <int D, bool DENSE>
static hipError_t launch_mode(const PagedAttnArgs& a, hipStream_t stream) {
  if (a.waves > 1) return launch_rows<D, DENSE, Codes4>(a, a.waves, a.join_groups, stream);
  const hipError_t e = a.token_waves == 8 ? launch_token<D, DENSE, 8>(a, stream) : launch_token<D, DENSE, 4>(a, stream);
  if (e != hipSuccess || a.ranges == 1) return e;
  paged_join_kernel<D, kJoinGroups><<<(int64_t)a.bh * a.lq, D / 4 * kJoinGroups, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, int d, bool dense, hipStream_t stream) {
  if (d == 128) return dense ? launch_mode<128, true>(a, stream) : launch_mode<128, false>(a, stream);
  return dense ? launch_mode<64, true>(a, stream) : launch_mode<64, false>(a, stream);
}

}  // namespace sparstar
