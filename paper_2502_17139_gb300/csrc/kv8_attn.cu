// fc_kv8_attn: verification attention over the paged 8-bit cache, and the
// weight that each cached token received.
#include <algorithm>
#include <cmath>

#include "kv8.cuh"
#include "kv8_attn.cuh"

FC_DEFINE_ERROR_WORD(kv8_attn)

namespace {

constexpr int HD = KV8_D;

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A warp a query row (request, node, head), four dimensions a lane, a key at a time.
__global__ void __launch_bounds__(256) k_kv8_attn_rows(Kv8Args a) {
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (row >= (long long)a.B * a.n_pad * a.H) return;
  const int h = (int)(row % a.H), i = (int)(row / a.H % a.n_pad), b = (int)(row / a.H / a.n_pad), gh = h / a.G;
  int kvl = a.kv_len[b], nn = a.n_nodes ? a.n_nodes[b] : a.n_pad;
  if (nn < 0 || nn > a.n_pad || kvl < 0 || kvl > (long long)a.max_pages << a.shift) {
    if (h == 0 && i == 0 && lane == 0) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_INVALID);
    nn = kvl = 0;
  }
  uint2* out = reinterpret_cast<uint2*>(a.out + row * HD) + lane;
  if (i >= nn) {
    *out = make_uint2(0, 0);
    return;
  }
  const int r = i * a.G + h - gh * a.G;
  auto four = [](const uint2& w) {
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u));
  };
  const float4 q = four(reinterpret_cast<const uint2*>(a.q + row * HD)[lane]);
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  float m = -INFINITY, l = 0.f;
  auto take = [&](const float4& k, const float4& v) {
    float z = fmaf(q.x, k.x, fmaf(q.y, k.y, fmaf(q.z, k.z, q.w * k.w)));
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) z += __shfl_xor_sync(0xFFFFFFFFu, z, x);
    z *= a.scale_log2;
    if (!(z <= m)) {
      const float mn = z, al = exp2_fast(m - mn);
      m = mn;
      l *= al;
      o.x *= al, o.y *= al, o.z *= al, o.w *= al;
    }
    const float p = z == -INFINITY ? 0.f : exp2_fast(z - m);
    l += p;
    o.x = fmaf(p, v.x, o.x), o.y = fmaf(p, v.y, o.y), o.z = fmaf(p, v.z, o.z), o.w = fmaf(p, v.w, o.w);
    return z;
  };
  const int32_t* tab = a.table + (size_t)b * a.max_pages;
  float* zs = a.z ? a.z + (((size_t)b * a.Hkv + gh) * a.R + r) * a.z_stride : nullptr;
  for (int j = 0; j < kvl; ++j) {
    const int page = tab[j >> a.shift];
    float z = -INFINITY;
    if ((unsigned)page >= (unsigned)a.n_pages) {
      if (lane == 0) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_INVALID);
    } else {
      const size_t at = (((size_t)page * a.Hkv + gh) << a.shift) + (j & ((1 << a.shift) - 1));
      auto cached = [&](const uint8_t* c, const float* s) {
        const uint32_t w = reinterpret_cast<const uint32_t*>(c + at * HD)[lane];
        const float2 x = e4m3x2_floats(w & 0xFFFFu), y = e4m3x2_floats(w >> 16);
        const float by = s[at >> 4];
        return make_float4(x.x * by, x.y * by, y.x * by, y.y * by);
      };
      z = take(cached(a.kc, a.ks), cached(a.vc, a.vs));
    }
    if (zs && lane == 0) zs[j] = z;
  }
  if (a.k_new)
    for (int j = 0; j < nn; ++j) {
      const bool sees = a.mask ? (a.mask[((size_t)b * a.n_pad + i) * ((a.n_pad + 63) / 64) + (j >> 6)] >> (j & 63)) & 1 : j <= i;
      const size_t at = (((size_t)b * a.Hkv + gh) * a.n_pad + j) * HD;
      if (sees) take(four(reinterpret_cast<const uint2*>(a.k_new + at)[lane]), four(reinterpret_cast<const uint2*>(a.v_new + at)[lane]));
    }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  *out = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
  if (a.z && lane == 0) a.lse[((size_t)b * a.Hkv + gh) * a.R + r] = l == 0.f ? INFINITY : m + log2f(l);
}

// weight = decay * weight + the sum over a kv head's rows of 2^(score - log2 of
// the row's sum): the scores that the attention left, four keys a thread.
__global__ void __launch_bounds__(256) k_kv8_weights(Kv8Args a, float* __restrict__ weight, float decay) {
  const int unit = blockIdx.y, b = unit / a.Hkv, gh = unit - b * a.Hkv;
  int kvl = a.kv_len[b], nn = a.n_nodes ? a.n_nodes[b] : a.n_pad;
  if (nn < 0 || nn > a.n_pad || kvl < 0 || kvl > (long long)a.max_pages << a.shift) return;
  const int R = nn * a.G;
  const float* z0 = a.z + (size_t)unit * a.R * a.z_stride;
  const float* lse = a.lse + (size_t)unit * a.R;
  for (long long j = ((long long)blockIdx.x * 256 + threadIdx.x) * 4; j < kvl; j += (long long)gridDim.x * 1024) {
    const int page = a.table[(size_t)b * a.max_pages + (j >> a.shift)];
    if ((unsigned)page >= (unsigned)a.n_pages) continue;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int r = 0; r < R; ++r) {
      const float4 z = *reinterpret_cast<const float4*>(z0 + (size_t)r * a.z_stride + j);
      const float m = lse[r];
      sum.x += exp2_fast(z.x - m), sum.y += exp2_fast(z.y - m), sum.z += exp2_fast(z.z - m), sum.w += exp2_fast(z.w - m);
    }
    float* w = weight + (((size_t)page * a.Hkv + gh) << a.shift) + (j & ((1 << a.shift) - 1));
    const float* s = &sum.x;
    for (int u = 0; u < 4 && j + u < kvl; ++u) w[u] = decay == 0.f ? s[u] : fmaf(decay, w[u], s[u]);
  }
}

bool shape_ok(int n_pad, int H, int Hkv) {
  return n_pad >= 1 && n_pad <= FC_MAX_NODES && H >= 1 && Hkv >= 1 && H % Hkv == 0 && H / Hkv <= 16;
}

// bytes of the scores and of the rows' sums that the weights are made from
size_t score_bytes(long long batch, int n_pad, int H, long long keys) {
  const size_t rows = (size_t)batch * n_pad * H;
  return (rows * (size_t)keys * 4 + rows * 4 + 255) & ~(size_t)255;
}

}  // namespace

extern "C" size_t fc_kv8_attn_workspace(int batch, int n_pad, int H, int Hkv, int64_t weight_keys) {
  if (batch < 1 || !shape_ok(n_pad, H, Hkv) || weight_keys < 0 || (weight_keys && n_pad * (H / Hkv) > 16)) return 0;
  return 256 + (weight_keys ? score_bytes(batch, n_pad, H, weight_keys) : 0);
}

extern "C" fc_status fc_kv8_attn(const void* d_q, const fc_kv8_cache* cache, const int32_t* d_table, int max_pages,
                                 const int32_t* d_kv_len, const void* d_k_new, const void* d_v_new,
                                 const uint64_t* d_mask, const int32_t* d_n_nodes, int batch, int n_pad, int H,
                                 float scale, float* d_weight, float decay, void* d_out, void* d_ws, size_t ws_bytes,
                                 fc_stream stream) {
  FC_NVTX_RANGE();
  if (const fc_status st = fc_kv8_check(cache)) return st;
  if (batch < 0 || max_pages < 1 || !(scale > 0.f) || !std::isfinite(scale) || (d_weight && !std::isfinite(decay))) return FC_ERR_INVALID_ARG;
  if (!shape_ok(n_pad, H, cache->Hkv)) return FC_ERR_UNSUPPORTED;
  const int shift = kv8_page_shift(cache->page_size), G = H / cache->Hkv;
  if ((long long)batch * H * n_pad > 1ll << 30 || (long long)max_pages << shift > 0x7FFFFFFFll || (d_weight && n_pad * G > 16))
    return FC_ERR_UNSUPPORTED;
  if (batch == 0) return FC_OK;
  if (!d_q || !d_table || !d_kv_len || !d_out || !kv8_aligned(d_q, 16) || !kv8_aligned(d_out, 16) || !d_k_new != !d_v_new ||
      !kv8_aligned(d_k_new, 16) || !kv8_aligned(d_v_new, 16) || !kv8_aligned(d_mask, 8) || (d_ws && !kv8_aligned(d_ws, 256)))
    return FC_ERR_INVALID_ARG;
  Kv8Args a{static_cast<const __nv_bfloat16*>(d_q),
            static_cast<const uint8_t*>(cache->k_codes),
            static_cast<const uint8_t*>(cache->v_codes),
            static_cast<const float*>(cache->k_scale),
            static_cast<const float*>(cache->v_scale),
            d_table,
            d_kv_len,
            static_cast<const __nv_bfloat16*>(d_k_new),
            static_cast<const __nv_bfloat16*>(d_v_new),
            d_mask,
            d_n_nodes,
            static_cast<__nv_bfloat16*>(d_out),
            batch,
            n_pad,
            H,
            cache->Hkv,
            G,
            n_pad * G,
            max_pages,
            cache->n_pages,
            shift,
            scale * 1.4426950408889634f,
            nullptr,
            nullptr,
            (long long)max_pages << shift,
            fc_error_slot()};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (d_weight) {
    const size_t need = score_bytes(batch, n_pad, H, a.z_stride);
    if (!d_ws || ws_bytes < 256 + need) return FC_ERR_WORKSPACE;
    if (batch * cache->Hkv > 65535) return FC_ERR_UNSUPPORTED;
    a.z = reinterpret_cast<float*>(static_cast<unsigned char*>(d_ws) + ws_bytes / 256 * 256 - need);
    a.lse = a.z + (size_t)batch * n_pad * H * a.z_stride;
  }
  k_kv8_attn_rows<<<(unsigned)(((long long)batch * n_pad * H + 7) / 8), 256, 0, s>>>(a);
  if (d_weight) {
    const dim3 grid((unsigned)std::min<long long>((a.z_stride + 1023) / 1024, 1024), (unsigned)(batch * cache->Hkv));
    k_kv8_weights<<<grid, 256, 0, s>>>(a, d_weight, decay);
  }
  return FC_CHECK_LAUNCH();
}
