// The paged cache as the launchers and kernels see it.
#pragma once

#include <stdint.h>

namespace brisk {

struct KvView {
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* table;    // [B, max_pages]
  const int32_t* seq_len;  // [B]
  int64_t page_stride, slot_stride, head_stride;  // elements
  int32_t page_shift, n_pages, max_pages;
};

}  // namespace brisk
