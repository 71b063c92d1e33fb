// What the paged 8-bit cache's calls share (kv8.cu, kv8_evict.cu, kv8_attn.cu,
// kv8_attn_tc.cu).
//
// A block is 16 tokens of a page and one kv head.  Its numbers are e4m3, its
// scale a power of two s = 2^e: the smallest e >= -120 with max|x| <= 448 s.
// A power of two because e4m3 is a floating type: any other scale would leave
// its relative rounding (2^-4) as it is, while with powers of two a block that
// gets a larger scale keeps its numbers exactly, but for those that become
// subnormal, and attention can move scales between factors without rounding.
#pragma once

#include <cuda_fp8.h>

#include "fc_common.cuh"

constexpr int KV8_D = 128;      // the only head dimension
constexpr int KV8_BLOCK = 16;   // tokens a scale
constexpr int KV8_MIN_EXP = -120, KV8_MAX_EXP = 120;

// log2 of a supported page size (16 .. 256 tokens), else -1.
static inline int kv8_page_shift(int page_size) {
  for (int s = 4; s <= 8; ++s)
    if (page_size == 1 << s) return s;
  return -1;
}

// The status of a cache description (kv8.cu).
fc_status fc_kv8_check(const fc_kv8_cache* c);

static inline bool kv8_aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Two e4m3 bytes (the low 16 bits) to floats; exact.
__device__ __forceinline__ float2 e4m3x2_floats(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return __half22float2(__half2(h));
}
// Two floats to e4m3 bytes, a the low one; nearest, ties to even, |x| > 448 to 448.
__device__ __forceinline__ uint32_t floats_e4m3x2(float a, float b) {
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ float kv8_pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
// The exponent of a scale (a power of two between 2^-126 and 2^127).
__device__ __forceinline__ int kv8_exp(float s) { return (int)((__float_as_uint(s) >> 23) & 255u) - 127; }
__device__ __forceinline__ bool kv8_nan(float s) { return !(s == s); }

// The smallest e with top <= 448 * 2^e = 1.75 * 2^(e + 8), top a finite
// magnitude (0 and subnormal numbers give a small e, for the caller to clamp).
__device__ __forceinline__ int kv8_exp_for(float top) {
  const uint32_t u = __float_as_uint(top);
  return (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
}

// Two e4m3 numbers (the low 16 bits) as fp16; exact.
__device__ __forceinline__ __half2 e4m3x2_halves(uint32_t two) {
  return __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3));
}
// Four e4m3 numbers times f, a power of two from 2^-24 to 2^15 in fp16 or 2^-24
// for any smaller one, rounded again; products of at most 448.  What fp16 rounds
// of its subnormal numbers is below 2^-14, nothing to e4m3's 2^-10.
__device__ __forceinline__ uint32_t kv8_times4(uint32_t w, __half2 f) {
  auto two = [&](uint32_t x) {
    return (uint32_t)__nv_cvt_halfraw2_to_fp8x2(static_cast<__half2_raw>(__hmul2(e4m3x2_halves(x), f)), __NV_SATFINITE, __NV_E4M3);
  };
  return two(w & 0xFFFFu) | (two(w >> 16) << 16);
}
__device__ __forceinline__ __half2 kv8_half_pow2(int d) { return __float2half2_rn(kv8_pow2(min(max(d, -24), 15))); }
// Four e4m3 numbers times 2^d, any d, rounded again; products of at most 448.
__device__ __forceinline__ uint32_t kv8_rescale4(uint32_t w, int d) {
  const float f = kv8_pow2(min(max(d, -31), 31));
  const float2 a = e4m3x2_floats(w & 0xFFFFu), b = e4m3x2_floats(w >> 16);
  return floats_e4m3x2(a.x * f, a.y * f) | (floats_e4m3x2(b.x * f, b.y * f) << 16);
}
