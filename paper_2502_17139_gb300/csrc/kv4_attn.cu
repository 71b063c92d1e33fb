// fc_kv4_attn: verification attention over the paged 4-bit cache.
#include <algorithm>
#include <cmath>

#include "fc_common.cuh"
#include "kv4.cuh"

FC_DEFINE_ERROR_WORD(kv4_attn)

namespace {

constexpr int HD = KV4_D;

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

// One warp a query row, one key at a time, four dimensions a lane.
__global__ void __launch_bounds__(128) k_kv4_attn_row(Kv4Args a) {
  const int lane = threadIdx.x & 31;
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= (long long)a.B * a.n_pad * a.H) return;
  const int h = (int)(row % a.H), i = (int)(row / a.H % a.n_pad), b = (int)(row / a.H / a.n_pad), g = h / a.G;
  const int kvl = a.kv_len[b], nn = a.n_nodes ? a.n_nodes[b] : a.n_pad;
  const bool bad = nn < 0 || nn > a.n_pad || kvl < 0 || kvl > (long long)a.max_pages << a.shift;
  if (bad && lane == 0) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_INVALID);
  auto f4 = [](const __nv_bfloat16* p, float (&v)[4]) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xFFFF0000u);
    v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xFFFF0000u);
  };
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f};
  f4(a.q + row * HD + 4 * lane, q);
  float m = -INFINITY, l = 0.f;
  auto key = [&](const float (&k)[4], const float (&v)[4]) {
    float s = q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3];
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, x);
    s *= a.scale_log2;
    const float mn = fmaxf(m, s), al = exp2f(m - mn), p = exp2f(s - mn);
    l = l * al + p;
#pragma unroll
    for (int x = 0; x < 4; ++x) o[x] = o[x] * al + p * v[x];
    m = mn;
  };
  if (!bad && i < nn) {
    for (int j = 0; j < kvl; ++j) {
      const int id = a.table[(size_t)b * a.max_pages + (j >> a.shift)];
      if (id < 0 || id >= a.n_pages) {
        if (lane == 0) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_INVALID);
        continue;
      }
      const size_t r = (((size_t)id * a.Hkv + g) << a.shift) + (j & ((1 << a.shift) - 1));
      const float ks = __bfloat162float(a.ks[r]), vs = __bfloat162float(a.vs[r]);
      const uint32_t kb = *reinterpret_cast<const uint16_t*>(a.kc + r * KV4_ROW + 2 * lane);
      const uint32_t vb = *reinterpret_cast<const uint16_t*>(a.vc + r * KV4_ROW + 2 * lane);
      float k[4], v[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        k[x] = (float)((int)((kb >> (4 * x)) & 15u) - 8) * ks;
        v[x] = (float)((int)((vb >> (4 * x)) & 15u) - 8) * vs;
      }
      key(k, v);
    }
    const int words = (a.n_pad + 63) / 64;
    for (int j = 0; a.k_new && j < nn; ++j) {
      const bool sees = a.mask ? (a.mask[((size_t)b * a.n_pad + i) * words + (j >> 6)] >> (j & 63)) & 1 : j <= i;
      if (!sees) continue;
      const size_t r = ((size_t)b * a.Hkv + g) * a.n_pad + j;
      float k[4], v[4];
      f4(a.k_new + r * HD + 4 * lane, k);
      f4(a.v_new + r * HD + 4 * lane, v);
      key(k, v);
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  *reinterpret_cast<uint2*>(a.out + row * HD + 4 * lane) =
      make_uint2(pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv));
}

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

bool shape_ok(int n_pad, int H, int Hkv) {
  return n_pad >= 1 && n_pad <= FC_MAX_NODES && H >= 1 && Hkv >= 1 && H % Hkv == 0 && H / Hkv <= 16;
}

}  // namespace

extern "C" size_t fc_kv4_attn_workspace(int batch, int n_pad, int H, int Hkv) {
  if (batch < 1 || !shape_ok(n_pad, H, Hkv)) return 0;
  return 256;
}

extern "C" fc_status fc_kv4_attn(const void* d_q, const fc_kv4_cache* cache, const int32_t* d_table, int max_pages,
                                 const int32_t* d_kv_len, const void* d_k_new, const void* d_v_new,
                                 const uint64_t* d_mask, const int32_t* d_n_nodes, int batch, int n_pad, int H,
                                 float scale, void* d_out, void* d_ws, size_t ws_bytes, fc_stream stream) {
  FC_NVTX_RANGE();
  if (const fc_status st = fc_kv4_check(cache)) return st;
  if (batch < 0 || max_pages < 1 || !(scale > 0.f) || !std::isfinite(scale)) return FC_ERR_INVALID_ARG;
  if (!shape_ok(n_pad, H, cache->Hkv)) return FC_ERR_UNSUPPORTED;
  if (batch == 0) return FC_OK;
  if (!d_q || !d_table || !d_kv_len || !d_out || !aligned(d_q, 16) || !aligned(d_out, 16) || !d_k_new != !d_v_new ||
      !aligned(d_k_new, 16) || !aligned(d_v_new, 16) || (d_ws && !aligned(d_ws, 256)))
    return FC_ERR_INVALID_ARG;
  Kv4Args a{static_cast<const __nv_bfloat16*>(d_q),
            static_cast<const uint8_t*>(cache->k_codes),
            static_cast<const uint8_t*>(cache->v_codes),
            static_cast<const __nv_bfloat16*>(cache->k_scale),
            static_cast<const __nv_bfloat16*>(cache->v_scale),
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
            H / cache->Hkv,
            max_pages,
            cache->n_pages,
            kv4_page_shift(cache->page_size),
            scale * 1.4426950408889634f,
            fc_error_slot()};
  const long long rows = (long long)batch * n_pad * H;
  if ((rows + 3) / 4 > 0x7FFFFFFFll) return FC_ERR_UNSUPPORTED;
  k_kv4_attn_row<<<(unsigned)((rows + 3) / 4), 128, 0, static_cast<cudaStream_t>(stream)>>>(a);
  return FC_CHECK_LAUNCH();
}
