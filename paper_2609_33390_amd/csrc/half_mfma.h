// Matrix instructions on the 2-byte types a cache may hold.
#pragma once

#include <utility>

#include "kv_common.h"

namespace brisk {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

// c + A B for A [32, 16] and B [16, 32]: lane l holds elements 8 (l / 32) .. + 7
// of row (column) l % 32 of A (B); register r of c is row 8 (r / 4) + 4 (l / 32) + r % 4,
// column l % 32.
template <bool F16>
__device__ __forceinline__ floatx16 mfma32(uint4 a, uint4 b, floatx16 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Two numbers rounded to the type, the first in the low half.
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  if constexpr (F16) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, h2{static_cast<_Float16>(lo), static_cast<_Float16>(hi)});
  } else {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, b2{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
  }
}

__device__ __forceinline__ float swap16_max(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float swap32_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Rows of keys or queries in LDS are RB bytes, their 16-byte chunks permuted
// by the row so that the b128 reads of one chunk of 16 rows meet in no bank.
template <int RB>
__device__ __forceinline__ int row_swizzle(int row) { return RB == 256 ? row & 15 : (row >> 1) & 7; }

// The address offset of the key that this lane copies in copy I of a
// wavefront, from the lane that holds it.  A copy is 1 KiB: 16 lanes a key for
// RB = 256 (lane 16 g + I holds key g of copy I), 8 for RB = 128 (lane
// 16 g + 2 I + x holds key 2 g + x).
template <int RB, int I>
__device__ __forceinline__ int64_t held_offset(int64_t at) {
  const int lo = static_cast<int>(at), hi = static_cast<int>(at >> 32);
  int l, h;
  if constexpr (RB == 256) {
    l = __builtin_amdgcn_update_dpp(0, lo, 0x150 + I, 0xF, 0xF, false);  // row_newbcast
    h = __builtin_amdgcn_update_dpp(0, hi, 0x150 + I, 0xF, 0xF, false);
  } else {
    l = __builtin_amdgcn_update_dpp(0, lo, 0x150 + 2 * I, 0xF, 0x3, false);  // lanes 0-7 of a row
    h = __builtin_amdgcn_update_dpp(0, hi, 0x150 + 2 * I, 0xF, 0x3, false);
    l = __builtin_amdgcn_update_dpp(l, lo, 0x150 + 2 * I + 1, 0xF, 0xC, false);  // lanes 8-15
    h = __builtin_amdgcn_update_dpp(h, hi, 0x150 + 2 * I + 1, 0xF, 0xC, false);
  }
  return static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(h)) << 32 | static_cast<uint32_t>(l));
}

// The key, within a wavefront's copies, whose offset this lane holds.
template <int RB>
__device__ __forceinline__ int held_key(int lane) {
  return RB == 256 ? lane % 16 * 4 + lane / 16 : lane % 16 / 2 * 8 + lane / 16 * 2 + lane % 2;
}

// Sixteen bytes a lane from global memory to LDS, to `dst` + 16 * lane (dst
// the same in all lanes).  Written as assembly because the compiler waits for
// every copy it knows of before any LDS read, and so would not let the copies
// of one tile fly while another is read; copies_landed() is the wait.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // m0 is reserved, so naming it as clobbered is noted
__device__ __forceinline__ void copy_to_lds(const void* src, void* dst) {
  const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) void*)dst));
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(__builtin_amdgcn_readfirstlane(at)), "v"(src)
               : "memory", "m0");
}
#pragma clang diagnostic pop

// Waits for the wavefront's own copies.
__device__ __forceinline__ void copies_landed() {
  __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (15 << 8));  // vmcnt(0)
  asm volatile("" ::: "memory");
}

// fn(integral_constant<int, 0>), ..., fn(integral_constant<int, N - 1>)
template <int N, class Fn>
__device__ __forceinline__ void each_index(Fn fn) {
  [&]<int... I>(std::integer_sequence<int, I...>) { (fn(std::integral_constant<int, I>{}), ...); }(
      std::make_integer_sequence<int, N>{});
}

// Source of LDS chunks that hold nothing.
__device__ const uint4 g_zeros[1] = {};

}  // namespace brisk
