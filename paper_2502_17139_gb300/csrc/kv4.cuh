// What the paged 4-bit cache's calls share (kv4.cu, kv4_attn.cu).
#pragma once

#include "fc_common.cuh"

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

// An attention workspace begins with counters that are zero between calls; what
// is written past them needs no such care, so that one workspace serves every
// shape.
constexpr size_t KV4_WS_COUNTERS = 1280;

// What an attention launch passes to its kernels.
struct Kv4Args {
  const __nv_bfloat16* q;
  const uint8_t *kc, *vc;
  const __nv_bfloat16 *ks, *vs;
  const int32_t* table;
  const int32_t* kv_len;
  const __nv_bfloat16 *k_new, *v_new;
  const uint64_t* mask;
  const int32_t* n_nodes;
  __nv_bfloat16* out;
  int B, n_pad, H, Hkv, G, max_pages, n_pages, shift;
  float scale_log2;
  unsigned int* err;
};

// A total cost cut into n shares of equal size (the first rem one longer), of
// at least `least` each unless there is less.
struct Kv4Cut {
  int n, q, rem;
  __device__ __forceinline__ Kv4Cut(int total, int grid, int least) {
    n = max(1, min(grid, total / least));
    q = total / n;
    rem = total - q * n;
  }
  __device__ __forceinline__ int start(int c) const { return c * q + min(c, rem); }
  __device__ __forceinline__ int share_of(int x) const {
    const int longer = rem * (q + 1);
    return x < longer ? x / (q + 1) : rem + (x - longer) / q;
  }
};

// The kernel for many query rows a kv head (kv4_attn_tc.cu).
size_t kv4_attn_many_workspace(int batch, int n_pad, int H, int Hkv);
fc_status kv4_attn_many(const Kv4Args& a, void* ws, size_t ws_bytes, cudaStream_t s);
