// The 8-bit key/value cache: quantising writes and exact reads.
//
// A cache holds e4m3 codes [BH, cap, D] and one scale byte e + 127 per block of
// tokens and head, [BH, ceil(cap / block)]; a value is code * 2^e.  Scales are powers
// of two, so that scaling rounds nothing: a code is the value's nearest e4m3 number
// (4 significant bits, half a step is 2^-4 of the value) and code * 2^e is exact in
// bf16.  e is the least integer with amax 2^-e <= 448, the largest e4m3 number, so the
// top binade is used whole; a free fp32 scale would gain less than one binade at the
// small end of a range of 17.
//
// Both kernels stream and are bound by memory: the write reads 2 bytes and writes 1 per
// element, the read the reverse.  24 heads, D = 128, K and V: 11,520 tokens written in 37 us
// (5.7 TB/s, some of it from the last-level cache), 84,032 read in 256 us (6.0 TB/s; a large
// copy reaches 4.95); one token 7.6 us and 300 tokens read 10.7, which is the call itself.
#include "device_common.h"

namespace sparstar {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Work-groups are launched in rows of at most this many: a launch may have fewer than 2^32
// threads along each axis.  (A loop over the rest in each of 65,536 work-groups took 299 us for
// the 84,032 tokens above, and 3% more for the 11,520.)
constexpr int64_t kCacheGridRow = 1 << 20;
static dim3 cache_grid(int64_t n) {
  const int64_t rows = (n + kCacheGridRow - 1) / kCacheGridRow;
  return dim3((uint32_t)((n + rows - 1) / rows), (uint32_t)rows);
}
__device__ __forceinline__ int64_t cache_group() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// 2^e of a scale byte: the byte is the exponent field of the float
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// four values -> four e4m3 codes (nearest even).  Infinities, and what would round past
// `most`, saturate there; NaN stays NaN.
__device__ __forceinline__ uint32_t pack4_e4m3(float a, float b, float c, float d, float most) {
  auto sat = [most](float x) { return x != x ? x : fminf(fmaxf(x, -most), most); };
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(sat(a), sat(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(sat(c), sat(d), r, true);
}

// One work-group per (K or V, batch * head, block that the new tokens touch).  The
// block's new rows are read once into registers (16 bytes per thread and row chunk),
// their largest finite magnitude gives the scale, and the codes go out.  Rows of the
// block from before keep their values: they hold the scale up, and are rounded again
// where the new rows raise it.
template <int D, int BLK>
__global__ __launch_bounds__(256) void cache_write_kernel(CacheWriteArgs a) {
  constexpr int CPR = D / 8, N = BLK * CPR / 256;  // 8-value chunks per row, per thread
  __shared__ float red[4];
  int64_t w = cache_group();
  if (w >= 2 * (int64_t)a.bh * a.n_blocks) return;
  const int blk_i = (int)(w % a.n_blocks);
  w /= a.n_blocks;
  const int64_t bh = w % a.bh;
  const bool is_v = w >= a.bh;
  const int64_t b = bh / a.heads;
  int64_t start = a.starts != nullptr ? a.starts[b] : a.start, count = a.l;
  if (a.counts != nullptr) count = a.counts[b] < a.l ? a.counts[b] : a.l;
  // rows outside [0, cap) do not exist: the tokens that would go there are dropped
  const int64_t lo = start > 0 ? start : 0, end = start + count < a.cap ? start + count : a.cap;
  const int64_t blk = lo / BLK + blk_i, row0 = blk * BLK;
  const int64_t first = lo > row0 ? lo : row0;  // the block's first new row
  if (first >= end || row0 >= end) return;
  const uint16_t* src = (is_v ? a.v : a.k) + (bh * a.l - start) * D;
  uint8_t* codes = (is_v ? a.v_cache : a.k_cache) + bh * a.cap * D;
  uint8_t* scale = (is_v ? a.v_scale : a.k_scale) + bh * ((a.cap + BLK - 1) / BLK) + blk;

  uint4 x[N];
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = threadIdx.x + 256 * i;
    const int64_t row = row0 + c / CPR;
    x[i] = make_uint4(0, 0, 0, 0);
    if (row >= first && row < end) x[i] = *reinterpret_cast<const uint4*>(src + row * D + 8 * (c % CPR));
    const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = fabsf(bf16_lo(u[e])), q = fabsf(bf16_hi(u[e]));
      if (p < INFINITY) amax = fmaxf(amax, p);
      if (q < INFINITY) amax = fmaxf(amax, q);
    }
  }
#pragma unroll
  for (int s = 32; s > 0; s /= 2) amax = fmaxf(amax, __shfl_xor(amax, s));
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = amax;
  __syncthreads();
  amax = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  // amax = m 2^x with 1/2 <= m < 1, and 448 = 7/8 2^9
  int e = kCacheExpMin;
  if (amax > 0.f) {
    e = __builtin_amdgcn_frexp_expf(amax) - (__builtin_amdgcn_frexp_mantf(amax) <= 0.875f ? 9 : 8);
    e = e < kCacheExpMin ? kCacheExpMin : (e > kCacheExpMax ? kCacheExpMax : e);
  }
  if (first > row0) {
    int held = (int)*scale - 127;
    held = held < kCacheExpMin ? kCacheExpMin : (held > kCacheExpMax ? kCacheExpMax : held);
    if (held < e) {
      const float f = __builtin_amdgcn_ldexpf(1.f, held - e);
      const int n = (int)(first - row0) * (D / 4);
      uint32_t* old = reinterpret_cast<uint32_t*>(codes + row0 * D);
      for (int i = threadIdx.x; i < n; i += 256) {
        const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(old[i], 1.f, false);
        const bf16x2 q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(old[i], 1.f, true);
        old[i] = pack4_e4m3((float)p[0] * f, (float)p[1] * f, (float)q[0] * f, (float)q[1] * f, 448.f);
      }
    } else {
      e = held;
    }
    __syncthreads();  // every thread has read the held scale
  }
  if (threadIdx.x == 0) *scale = (uint8_t)(e + 127);
  const float inv = __builtin_amdgcn_ldexpf(1.f, -e);
  // (256 * 2^120 is past the largest bf16 number)
  const float most = e == kCacheExpMax ? 240.f : 448.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = threadIdx.x + 256 * i;
    const int64_t row = row0 + c / CPR;
    if (row < first || row >= end) continue;
    const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
    uint2 r;
    r.x = pack4_e4m3(bf16_lo(u[0]) * inv, bf16_hi(u[0]) * inv, bf16_lo(u[1]) * inv, bf16_hi(u[1]) * inv, most);
    r.y = pack4_e4m3(bf16_lo(u[2]) * inv, bf16_hi(u[2]) * inv, bf16_lo(u[3]) * inv, bf16_hi(u[3]) * inv, most);
    *reinterpret_cast<uint2*>(codes + row * D + 8 * (c % CPR)) = r;
  }
}

// One thread per 16 codes.
__global__ __launch_bounds__(256) void cache_read_kernel(CacheReadArgs a) {
  const int64_t cpr = a.d / 16, per_bh = a.l * cpr, n = (int64_t)a.bh * per_bh;
  int64_t i = cache_group() * 256 + threadIdx.x;
  // the first n threads take K where it is wanted, the next n (or the first) V
  const bool is_v = a.k_out == nullptr || i >= n;
  if (a.k_out != nullptr && is_v) i -= n;
  if (i >= n || (is_v && a.v_out == nullptr)) return;
  const int64_t bh = i / per_bh, r = i - bh * per_bh;
  const int64_t row = a.start + r / cpr;
  const uint8_t* codes = (is_v ? a.v_cache : a.k_cache) + (bh * a.cap + row) * a.d + 16 * (r % cpr);
  const float sc = scale_of((is_v ? a.v_scale : a.k_scale)[bh * ((a.cap + a.block - 1) / a.block) + row / a.block]);
  const uint4 u = *reinterpret_cast<const uint4*>(codes);
  auto two = [&](uint32_t x, uint32_t& lo, uint32_t& hi) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, sc, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, sc, true));
  };
  uint4 p, q;
  two(u.x, p.x, p.y);
  two(u.y, p.z, p.w);
  two(u.z, q.x, q.y);
  two(u.w, q.z, q.w);
  uint4* out = reinterpret_cast<uint4*>((is_v ? a.v_out : a.k_out) + 16 * i);
  out[0] = p;
  out[1] = q;
}

hipError_t launch_cache_write(const CacheWriteArgs& a, int d, int block, hipStream_t stream) {
  const dim3 grid = cache_grid(2 * (int64_t)a.bh * a.n_blocks);
  if (d == 128 && block == 64) cache_write_kernel<128, 64><<<grid, 256, 0, stream>>>(a);
  else if (d == 128) cache_write_kernel<128, 128><<<grid, 256, 0, stream>>>(a);
  else if (block == 64) cache_write_kernel<64, 64><<<grid, 256, 0, stream>>>(a);
  else cache_write_kernel<64, 128><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_read(const CacheReadArgs& a, hipStream_t stream) {
  const int64_t n = (int64_t)a.bh * a.l * (a.d / 16) * ((a.k_out != nullptr) + (a.v_out != nullptr));
  cache_read_kernel<<<cache_grid((n + 255) / 256), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace sparstar
