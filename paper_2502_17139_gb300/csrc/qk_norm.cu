// fc_qk_norm_rope: RMSNorm of every query and key head and its rotation by
// position, in the pass that lays queries node-major and keys and values
// head-major, as the attention calls read them.
//
// A head's row of D values is held by LP lanes (the power of two from D / 16
// up), lane c the 8 values 8c.. and their partners D/2 + 8c.. : the sum of
// squares is a shuffle over LP lanes, the rotation needs no exchange, and the
// 8 sines and cosines of a lane's dimensions serve all heads of the row that the
// warp takes.  The read and the write bound it (rows * (H + 2 Hkv) * D * 4
// bytes; 65000 rows of 16 + 16 + 16 heads of 128 272 us, 5.9 TB/s, a copy's rate
// 6.6; 267 without the check of the squares' range; unrolled over heads or rows, with
// prefetches or streaming hints, and on other grids 278 to 387); fp32 inside,
// rounded once.  32 rows take 3.7 us, latency.
#include <algorithm>
#include <cmath>

#include "fc_common.cuh"

FC_DEFINE_ERROR_WORD(norm)

namespace {

constexpr int NR_THREADS = 256, NR_WARPS = NR_THREADS / 32;
constexpr int MAX_D = 512;
// Sums of squares that fp32 holds with all their parts: up to SS_MAX, and from
// SS_MIN on unless eps is as much (it then outweighs what is lost).
constexpr uint32_t SS_MAX = 0x7B800000u, SS_MIN = 0x17800000u;  // 2^120, 2^-80: fp32's bits, in the numbers' order

struct NormArgs {
  const __nv_bfloat16 *q, *k, *v;
  int64_t q_seq, q_row, q_head, kv_seq, kv_row, kv_head;  // strides in elements
  const __nv_bfloat16 *wq, *wk;
  const int32_t* pos;
  __nv_bfloat16 *q_out, *k_out, *v_out;
  int n, H, Hkv, D, heads, slices, per;  // heads: H + Hkv (+ Hkv with values); a warp takes `per` of them
  long long items;                       // rows * slices
  float eps;
  uint32_t ss_min;  // SS_MIN or 0
  double nl2f;  // -2 log2(base) / D
};

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

template <int LP>
__global__ void __launch_bounds__(NR_THREADS) k_qk_norm_rope(NormArgs a) {
  __shared__ float2 tab[MAX_D / 2];
  fc_rope_table(tab, a.D / 2, a.nl2f);
  __syncthreads();
  constexpr int AT_ONCE = 32 / LP;  // heads
  const int lane = threadIdx.x & 31, c = lane % LP, sub = lane / LP, chunks = a.D / 16;
  const bool on = c < chunks;
  for (long long it = (long long)blockIdx.x * NR_WARPS + (threadIdx.x >> 5); it < a.items; it += (long long)gridDim.x * NR_WARPS) {
    const long long row = it / a.slices;
    const int h0 = (int)(it - row * a.slices) * a.per, h1 = min(a.heads, h0 + a.per);
    const long long b = row / a.n;
    const int i = (int)(row - b * a.n);
    const int p = a.pos[row];
    float sn[8], cs[8];
    if (h0 < a.H + a.Hkv) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sn[j] = 0.f, cs[j] = 1.f;
        if (on && p >= 0) fc_rope_sincos((float)p, tab[8 * c + j], sn[j], cs[j]);
      }
    }
    for (int hh = h0; hh < h1; hh += AT_ONCE) {
      const int h = hh + sub;
      const bool in = on && h < h1;
      const bool query = h < a.H, value = h >= a.H + a.Hkv;
      const int g = query ? h : value ? h - a.H - a.Hkv : h - a.H;
      uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
      if (in) {
        const __nv_bfloat16* x = query ? a.q + b * a.q_seq + i * a.q_row + g * a.q_head
                                       : (value ? a.v : a.k) + b * a.kv_seq + i * a.kv_row + g * a.kv_head;
        lo = reinterpret_cast<const uint4*>(x)[c];
        hi = reinterpret_cast<const uint4*>(x)[c + chunks];
      }
      float ss = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const uint32_t l = (&lo.x)[u], m = (&hi.x)[u];
        ss = fmaf(lo_f(l), lo_f(l), fmaf(hi_f(l), hi_f(l), fmaf(lo_f(m), lo_f(m), fmaf(hi_f(m), hi_f(m), ss))));
      }
#pragma unroll
      for (int o = 1; o < LP; o <<= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
      float by = 1.f, eps = a.eps;
      if (__builtin_expect(__any_sync(0xFFFFFFFFu, __float_as_uint(ss) - a.ss_min > SS_MAX - a.ss_min), 0)) {  // once more, of x times a power of two
        by = !(ss <= __uint_as_float(SS_MAX)) ? 0x1p-80f : ss < __uint_as_float(a.ss_min) ? 0x1p100f : 1.f;
        ss = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t l = (&lo.x)[u], m = (&hi.x)[u];
          const float x0 = lo_f(l) * by, x1 = hi_f(l) * by, y0 = lo_f(m) * by, y1 = hi_f(m) * by;
          ss = fmaf(x0, x0, fmaf(x1, x1, fmaf(y0, y0, fmaf(y1, y1, ss))));
        }
#pragma unroll
        for (int o = 1; o < LP; o <<= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
        eps = eps * by * by;
      }
      if (!in) continue;
      if (!value) {
        const float inv = rsqrtf(ss / (float)a.D + eps) * by;
        const uint4* w = reinterpret_cast<const uint4*>(query ? a.wq : a.wk);
        const uint4 wl = w[c], wh = w[c + chunks];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t l = (&lo.x)[u], m = (&hi.x)[u], gl = (&wl.x)[u], gh = (&wh.x)[u];
          const float x0 = lo_f(l) * inv * lo_f(gl), x1 = hi_f(l) * inv * hi_f(gl);
          const float y0 = lo_f(m) * inv * lo_f(gh), y1 = hi_f(m) * inv * hi_f(gh);
          (&lo.x)[u] = pack_bf16x2(x0 * cs[2 * u] - y0 * sn[2 * u], x1 * cs[2 * u + 1] - y1 * sn[2 * u + 1]);
          (&hi.x)[u] = pack_bf16x2(y0 * cs[2 * u] + x0 * sn[2 * u], y1 * cs[2 * u + 1] + x1 * sn[2 * u + 1]);
        }
      }
      __nv_bfloat16* out = query ? a.q_out + (row * a.H + g) * a.D : (value ? a.v_out : a.k_out) + ((b * a.Hkv + g) * a.n + i) * a.D;
      reinterpret_cast<uint4*>(out)[c] = lo;
      reinterpret_cast<uint4*>(out)[c + chunks] = hi;
    }
  }
}

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

extern "C" fc_status fc_qk_norm_rope(const void* d_q, int64_t q_seq_stride, int64_t q_row_stride, int64_t q_head_stride,
                                     const void* d_k, const void* d_v, int64_t kv_seq_stride, int64_t kv_row_stride,
                                     int64_t kv_head_stride, const void* d_wq, const void* d_wk, const int32_t* d_pos,
                                     int batch, int n, int H, int Hkv, int D, float base, float eps, void* d_q_out,
                                     void* d_k_out, void* d_v_out, fc_stream stream) {
  FC_NVTX_RANGE();
  if (batch < 0 || n < 0 || H < 1 || Hkv < 1 || D < 16 || D % 16 || !(base > 0.f) || !std::isfinite(base) || !(eps >= 0.f) ||
      !std::isfinite(eps) || q_seq_stride < 0 || q_row_stride < 0 || q_head_stride < 0 || kv_seq_stride < 0 || kv_row_stride < 0 ||
      kv_head_stride < 0 || (q_seq_stride | q_row_stride | q_head_stride | kv_seq_stride | kv_row_stride | kv_head_stride) % 8)
    return FC_ERR_INVALID_ARG;
  if (D > MAX_D || H > 1 << 20 || Hkv > 1 << 20) return FC_ERR_UNSUPPORTED;
  if (batch == 0 || n == 0) return FC_OK;
  if (!d_q || !d_k || !d_wq || !d_wk || !d_pos || !d_q_out || !d_k_out || !d_v != !d_v_out || !aligned16(d_q) || !aligned16(d_k) ||
      !aligned16(d_v) || !aligned16(d_wq) || !aligned16(d_wk) || !aligned16(d_q_out) || !aligned16(d_k_out) || !aligned16(d_v_out))
    return FC_ERR_INVALID_ARG;
  auto bf = [](const void* p) { return static_cast<const __nv_bfloat16*>(p); };
  const long long rows = (long long)batch * n;
  const int heads = H + Hkv + (d_v ? Hkv : 0), lp = D <= 64 ? 4 : D <= 128 ? 8 : D <= 256 ? 16 : 32, at_once = 32 / lp;
  // few rows: as many warps as the row has groups of heads; many: a row a warp, whose sines serve all heads
  const int per = rows * ((heads + at_once - 1) / at_once) <= 152 * 64 ? at_once : heads, slices = (heads + per - 1) / per;
  NormArgs a{bf(d_q), bf(d_k), bf(d_v), q_seq_stride, q_row_stride, q_head_stride, kv_seq_stride, kv_row_stride, kv_head_stride,
             bf(d_wq), bf(d_wk), d_pos, static_cast<__nv_bfloat16*>(d_q_out), static_cast<__nv_bfloat16*>(d_k_out),
             static_cast<__nv_bfloat16*>(d_v_out), n, H, Hkv, D, heads, slices, per, rows * slices, eps, eps < 0x1p-80f ? SS_MIN : 0u,
             -2.0 * std::log2((double)base) / D};
  const unsigned grid = (unsigned)std::min<long long>((a.items + NR_WARPS - 1) / NR_WARPS, 152 * 8);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (lp == 4) k_qk_norm_rope<4><<<grid, NR_THREADS, 0, s>>>(a);
  else if (lp == 8) k_qk_norm_rope<8><<<grid, NR_THREADS, 0, s>>>(a);
  else if (lp == 16) k_qk_norm_rope<16><<<grid, NR_THREADS, 0, s>>>(a);
  else k_qk_norm_rope<32><<<grid, NR_THREADS, 0, s>>>(a);
  return FC_CHECK_LAUNCH();
}
