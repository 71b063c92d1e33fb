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
