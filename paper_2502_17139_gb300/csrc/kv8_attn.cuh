// What an attention launch over the 8-bit cache passes to its kernels.
#pragma once

#include "kv8.cuh"

struct Kv8Args {
  const __nv_bfloat16* q;
  const uint8_t *kc, *vc;
  const float *ks, *vs;
  const int32_t* table;
  const int32_t* kv_len;
  const __nv_bfloat16 *k_new, *v_new;
  const uint64_t* mask;
  const int32_t* n_nodes;
  __nv_bfloat16* out;
  int B, n_pad, H, Hkv, G, R, max_pages, n_pages, shift;  // R = n_pad * G: query rows a kv head, node-major
  float scale_log2;
  // for the weights (else z is NULL): [B][Hkv][R][z_stride] scores in base 2 and
  // [B][Hkv][R] their rows' log2 of the sum of powers (+infinity where no key is seen)
  float* z;
  float* lse;
  long long z_stride;
  unsigned int* err;
};

// A total cost cut into n shares of equal size (the first rem one longer), of
// at least `least` each unless there is less.
struct KvCut {
  int n, q, rem;
  __device__ __forceinline__ KvCut(int total, int grid, int least) {
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

// A workspace begins with counters that are zero between calls; what is written
// past them needs no such care, so that one workspace serves every shape.
constexpr size_t KV8_WS_COUNTERS = 4096;

// The kernel for many query rows a kv head (kv8_attn_tc.cu).
size_t kv8_attn_many_workspace(int batch, int n_pad, int H, int Hkv);
fc_status kv8_attn_many(const Kv8Args& a, void* ws, size_t ws_bytes, cudaStream_t s);
