// What the paged 4-bit cache's calls share (kv4.cu, kv4_attn.cu).
#pragma once

#include "../../include/fastcoder.h"

constexpr int KV4_D = 128;           // the only head dimension
constexpr int KV4_ROW = KV4_D / 2;   // bytes of a cached row's numbers

// log2 of a supported page size (16 .. 256 tokens), else -1.
static inline int kv4_page_shift(int page_size) {
  for (int s = 4; s <= 8; ++s)
    if (page_size == 1 << s) return s;
  return -1;
}

// The status of a cache description (kv4.cu).
fc_status fc_kv4_check(const fc_kv4_cache* c);
