// Matrix instructions on the 2-byte types a cache may hold.
#pragma once

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

// Rows of keys or queries in LDS are RB bytes, their 16-byte chunks permuted
// by the row so that the b128 reads of one chunk of 16 rows meet in no bank.
template <int RB>
__device__ __forceinline__ int row_swizzle(int row) { return RB == 256 ? row & 15 : (row >> 1) & 7; }

}  // namespace brisk
