// What the attention kernels share on the device: vector types, cross-half
// reductions, the LDS transpose read, and direct-to-LDS tile loads.
#pragma once

#include <type_traits>
#include <utility>

#include "device_common.h"

namespace sparstar {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float half_swap_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float half_swap_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ uint32_t pack2_bf16(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}

// B operand of 16-row k-step `half` of a 32-row sub-tile, of packed values
typedef uint32_t u32x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ bf16x8 pack_half(u32x8 pk, int half) {
  const u32x4 lo = __builtin_shufflevector(pk, pk, 0, 1, 2, 3), hi = __builtin_shufflevector(pk, pk, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, half == 0 ? lo : hi);
}

__device__ __forceinline__ s16x4 lds_read_tr(const uint16_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(const_cast<uint16_t*>(p)));
}

// Buffer descriptor as four dwords (raw buffer, stride 0, `bytes` records):
// the form the inline-asm direct-to-LDS load takes.
typedef int i32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ i32x4 raw_rsrc(const void* base, uint32_t bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  i32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)p);
  r[1] = __builtin_amdgcn_readfirstlane((int)((uint32_t)(p >> 32) & 0xffffu));
  r[2] = __builtin_amdgcn_readfirstlane((int)bytes);
  r[3] = 0x00020000;
  return r;
}

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return (uint32_t)reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) void*)p);
}

// Direct-to-LDS loads: lane l of a wave-wide load copies 16 bytes from
// buffer offset voff (+ the instruction offset) to LDS byte m0 (+ the same
// instruction offset) + 16 l.  Written as inline assembly so that the compiler
// does not order every later LDS read behind them; each caller waits for these
// loads explicitly (vmcnt) before a barrier makes the tile visible.
//
// A wave's share of one tile: N wave-wide loads after a single M0 write.  The
// instruction offset moves the LDS destination and the memory address alike,
// so load i goes to LDS m0 + 1024 i + 16 l and reads voff[i] + 1024 i (the
// callers pass voff[i] already reduced by 1024 i).
template <int N>
__device__ __forceinline__ void dma_tile(uint32_t m0, const uint32_t* voff, i32x4 rsrc) {
  static_assert(N == 1 || N == 2 || N == 4, "loads per wave and tile");
  if constexpr (N == 1) {
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %1, %2, 0 offen lds"
        :
        : "s"(m0), "v"(voff[0]), "s"(rsrc)
        : "memory", "m0");
  } else if constexpr (N == 2) {
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %1, %3, 0 offen lds\n\t"
        "buffer_load_dwordx4 %2, %3, 0 offen offset:0x400 lds"
        :
        : "s"(m0), "v"(voff[0]), "v"(voff[1]), "s"(rsrc)
        : "memory", "m0");
  } else {
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %1, %5, 0 offen lds\n\t"
        "buffer_load_dwordx4 %2, %5, 0 offen offset:0x400 lds\n\t"
        "buffer_load_dwordx4 %3, %5, 0 offen offset:0x800 lds\n\t"
        "buffer_load_dwordx4 %4, %5, 0 offen offset:0xc00 lds"
        :
        : "s"(m0), "v"(voff[0]), "v"(voff[1]), "v"(voff[2]), "v"(voff[3]), "s"(rsrc)
        : "memory", "m0");
  }
}

// s_waitcnt with only the vector-memory counter constrained (<= n outstanding)
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

// f(0), .., f(N - 1) with each index a compile-time constant
template <class F, int... I>
__device__ __forceinline__ void static_for(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
  static_for(f, std::make_integer_sequence<int, N>{});
}

}  // namespace sparstar
