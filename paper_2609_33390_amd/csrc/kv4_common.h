// Addressing and codes of the 4-bit paged cache.
//
// A head is held as z + s c: z its smallest element, s the step, c = 0 .. 15.
// The codes of a block of 16 slots lie as the matrix instructions take them, so
// that attention loads its operands from memory to registers, in lane order and
// without a pass through LDS.  With W the width (64 or 128), a block is
//   [0, 8 W)       keys: chunk (t, key), t = 0 .. 3, of W / 8 bytes at
//                  (16 t + key) W / 8; its word i holds elements
//                  t W / 4 + 8 i + e of the key, e at nibble e / 2 + 4 (e % 2),
//                  the word turned left by 3 bits
//   [8 W, 16 W)    values: chunk (t, x), x = 0 .. 15, of W / 8 bytes at
//                  (16 t + x) W / 8; its 16 bits 4 y + u hold slot 4 t + u, nibble
//                  j element x + 16 (4 y + j).  A slot's bits fill whole bytes, so
//                  slots are written without reading their neighbours
//   then 16 pairs (s, z) of 2-byte numbers of the keys, and 16 of the values.
// The turn by 3 puts each of a word's code pairs at bits 3 .. 6 of its halves
// with one shift: there, under the exponent of 16, a bf16 reads 16 + c.
#pragma once

#include "half_mfma.h"
#include "kv4_view.h"

namespace brisk {

// Slots of sequence b, cut to `most` (itself at most what the table addresses).
__device__ __forceinline__ int kv4_len(const Kv4View& c, int b, int most) { return min(max(c.seq_len[b], 0), most); }

// The block that holds slot j of sequence b, for head h; 0 <= j < max_pages << page_shift.
template <int W>
__device__ __forceinline__ uint8_t* kv4_block(const Kv4View& c, int b, int h, int j) {
  const int page = clamp_id(c.table[static_cast<int64_t>(b) * c.max_pages + (j >> c.page_shift)], c.n_pages);
  return c.pages + page * c.page_stride + h * c.head_stride +
         static_cast<int64_t>((j & ((1 << c.page_shift) - 1)) / kKv4Block) * kv4_block_bytes(W);
}

// The step (low half) and the lowest value (high half) of a pair.
template <bool F16>
__device__ __forceinline__ float kv4_step(uint32_t w) { return half_to_f32<F16>(w & 0xFFFF); }
template <bool F16>
__device__ __forceinline__ float kv4_low(uint32_t w) {
  return F16 ? half_to_f32<F16>(w >> 16) : __uint_as_float(w & 0xFFFF0000u);
}

}  // namespace brisk
