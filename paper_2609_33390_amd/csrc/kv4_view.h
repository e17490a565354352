// The 4-bit paged cache as the launchers and kernels see it.
#pragma once

#include <stdint.h>

namespace brisk {

// A head of D elements is held as one of `kv4_width(D)`, the elements past D as code 0.
// Blocks of 16 slots of a head lie one after the other in a page's part for that head.
constexpr int kKv4Block = 16;                                                   // slots
constexpr int kv4_width(int D) { return D <= 64 ? 64 : 128; }
constexpr int kv4_slot_bytes(int width) { return width + 8; }                   // codes and (step, lowest) of key and value
constexpr int kv4_block_bytes(int width) { return kKv4Block * kv4_slot_bytes(width); }

struct Kv4View {
  uint8_t* pages;
  const int32_t* table;    // [B, max_pages]
  const int32_t* seq_len;  // [B]
  int64_t page_stride, head_stride;  // bytes
  int32_t page_shift, n_pages, max_pages;
};

}  // namespace brisk
