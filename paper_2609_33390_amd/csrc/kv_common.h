// Addressing of the paged cache, and the 2-byte types it may hold.
#pragma once

#include "device_common.h"
#include "kv_view.h"

namespace brisk {

// Slots of sequence b, cut to `most` (itself at most what the table addresses).
__device__ __forceinline__ int kv_len(const KvView& c, int b, int most) {
  return min(max(c.seq_len[b], 0), most);
}

// First element of slot j of sequence b for head 0; 0 <= j < max_pages << page_shift.
__device__ __forceinline__ int64_t kv_slot(const KvView& c, int b, int j) {
  const int page = clamp_id(c.table[static_cast<int64_t>(b) * c.max_pages + (j >> c.page_shift)], c.n_pages);
  return page * c.page_stride + (j & ((1 << c.page_shift) - 1)) * c.slot_stride;
}

// Whether block position i sees the block's own position t; `row` is the
// position's mask word (all ones without a mask).
__device__ __forceinline__ bool block_sees(uint64_t row, int t) { return (row >> (t & 63)) & 1; }

template <bool F16>
__device__ __forceinline__ float half_to_f32(uint16_t b) {
  if constexpr (F16) return static_cast<float>(__builtin_bit_cast(_Float16, b));
  return bf16_to_f32(b);
}

// Round to nearest even.
template <bool F16>
__device__ __forceinline__ uint16_t f32_to_half(float x) {
  if constexpr (F16) return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
  return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
}

}  // namespace brisk
