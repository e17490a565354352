// The paged cache as the launchers and kernels see it.
#pragma once

#include <stdint.h>

namespace brisk {

// The 32-wide slices that the kernels take a head of D elements as, and the bytes
// of its keys and values in LDS.  Rows of LDS are 128 or 256 bytes, so a head of
// three slices ends before its row does: only a head that fills the row may be
// copied without asking of every 16-byte chunk whether the head has it.
constexpr int head_slices(int D) { return D <= 64 ? 2 : D <= 96 ? 3 : 4; }
constexpr int lds_row_bytes(int slices) { return slices > 2 ? 256 : 128; }
constexpr bool head_fills_row(int D, int slices) { return 2 * D == lds_row_bytes(slices); }

struct KvView {
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* table;    // [B, max_pages]
  const int32_t* seq_len;  // [B]
  int64_t page_stride, slot_stride, head_stride;  // elements
  int32_t page_shift, n_pages, max_pages;
};

}  // namespace brisk
