// Products of a few rows with weights in 4 bits (fc_w4_pack, fc_w4_matvec):
//   y[m][n] = sum over groups t of s[t][n] * sum_{k in group t} x[m][k] c[k][n],
// c whole numbers in -7..7, s bf16 scales (fastcoder.h has the quantisation).
//
// Weights are packed so that a warp's 16-byte loads are tensor-core operands.
// A tile holds 16 columns x 64 k, 512 bytes, lane (g = lane / 4, t = lane % 4)
// owning 16 of them: word w (k-step w of the tile) has in nibble i (i < 4) the
// first and in nibble i + 4 the second element of operand register i of
// mma.m16n8k16, whose rows are the columns g and g + 8 of the tile
// (registers 0, 2 and 1, 3).  The k of k-step w are 32 (w / 2) + 8 t +
// 4 (w % 2) + {0, 1} (registers 0, 1) and + {2, 3} (registers 2, 3), so that a
// lane's part of x is 8 values in a row, one 16-byte load for two k-steps, and
// no k-step crosses a group of 32.  Tiles run over k first.
#include <algorithm>

#include "fc_common.cuh"

namespace {

constexpr int TK = 64;           // k a tile
constexpr int TN = 16;           // columns a tile
constexpr int TILE_BYTES = 512;
constexpr int MV_WARPS = 8;

// (k in the tile, column in the tile) of element e (0 or 1) of register i of
// k-step w in lane (g, t)
__host__ __device__ constexpr int elem_k(int w, int t, int i, int e) {
  return 32 * (w >> 1) + 8 * t + 4 * (w & 1) + 2 * (i >> 1) + e;
}
__host__ __device__ constexpr int elem_n(int g, int i) { return g + 8 * (i & 1); }

// bf16 scale of a largest magnitude given as bf16 bits without the sign
__device__ __forceinline__ __nv_bfloat16 scale_of(uint32_t top) {
  return top >= 0x7F80u ? __ushort_as_bfloat16(0x7FC0)
                        : __float2bfloat16_rn(__fdiv_rn(__uint_as_float(top << 16), 7.f));
}

// One thread a (group, column); consecutive threads take consecutive columns.
__global__ void k_w4_scale(const uint16_t* __restrict__ w, int K, int N, int group, __nv_bfloat16* __restrict__ s) {
  const size_t items = (size_t)(K / group) * N;
  for (size_t e = blockIdx.x * (size_t)blockDim.x + threadIdx.x; e < items; e += (size_t)gridDim.x * blockDim.x) {
    const size_t t = e / N, n = e - t * N;
    uint32_t top = 0;
    for (int k = 0; k < group; ++k) top = std::max<uint32_t>(top, w[(t * group + k) * N + n] & 0x7FFFu);
    s[e] = scale_of(top);
  }
}

// One warp a tile; columns past N are packed as zeros (number 0).
__global__ void k_w4_pack(const __nv_bfloat16* __restrict__ w, int K, int N, int group,
                          const __nv_bfloat16* __restrict__ s, uint4* __restrict__ out) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int kt = K / TK;
  const long long tiles = (long long)((N + TN - 1) / TN) * kt;
  const long long stride = (long long)gridDim.x * (blockDim.x >> 5);
  for (long long i = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); i < tiles; i += stride) {
    const int nt = (int)(i / kt), k0 = (int)(i - (long long)nt * kt) * TK;
    uint4 v;
    uint32_t* vw = &v.x;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      uint32_t word = 0;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int n = nt * TN + elem_n(g, r);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int k = k0 + elem_k(x, t, r, e);
          int c = 0;
          if (n < N) {
            const float sc = __bfloat162float(s[(size_t)(k / group) * N + n]);
            const float q = __fdiv_rn(__bfloat162float(w[(size_t)k * N + n]), sc);
            if (sc > 0.f) c = (int)fminf(fmaxf(rintf(q), -7.f), 7.f);
          }
          word |= (uint32_t)(c + 8) << (4 * (r + 4 * e));
        }
      }
      vw[x] = word;
    }
    out[i * 32 + lane] = v;
  }
}

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1, const float (&c)[4]) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}

// Two numbers of a packed word as bf16: 0x4300 | c is 128 + c, that is 136
// more than the number.  The surplus, 136 times the sum of x over the tile,
// comes off through the accumulators' starting value.
__device__ __forceinline__ uint32_t two(uint32_t w, int i) { return ((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u; }

constexpr uint32_t MINUS_136 = 0xC308C308u;  // two bf16 values

// A CTA takes MT tiles of columns, its warps every MV_WARPS-th tile of k; the
// warps' sums meet in shared memory.  NT: 8-row tiles of x.  STEPS: k-steps
// that share a scale (the group, or the whole tile).
template <int MT, int NT, int STEPS>
__global__ void __launch_bounds__(MV_WARPS * 32) k_w4_matvec(const uint4* __restrict__ x, const uint4* __restrict__ codes,
                                                             const __nv_bfloat16* __restrict__ scale, int M, int K,
                                                             int N, int gshift, __nv_bfloat16* __restrict__ y) {
  __shared__ float s_sum[MV_WARPS][MT * TN][NT * 8 + 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int kt = K / TK, n0 = blockIdx.x * (MT * TN), n_tiles = (N + TN - 1) / TN;
  float acc[MT][NT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.f;
#pragma unroll 2
  for (int j = warp; j < kt; j += MV_WARPS) {
    uint4 cw[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int tile = blockIdx.x * MT + m;
      cw[m] = tile < n_tiles ? codes[((size_t)tile * kt + j) * 32 + lane] : make_uint4(0, 0, 0, 0);
    }
    uint4 xv[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int row = n * 8 + g;
#pragma unroll
      for (int p = 0; p < 2; ++p)
        xv[n][p] = row < M ? x[((size_t)row * K + j * TK + 32 * p) / 8 + t] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int w0 = 0; w0 < 4; w0 += STEPS) {
      float sc[MT][2];
      const size_t grp = (size_t)((j * TK + w0 * 16) >> gshift) * N;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int n = n0 + m * TN + g + 8 * i;
          sc[m][i] = n < N ? __bfloat162float(scale[grp + n]) : 0.f;
        }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
        float off[4];
#pragma unroll
        for (int w = w0; w < w0 + STEPS; ++w) {
          const uint32_t* xw = &xv[n][w >> 1].x;
          if (w == w0) mma_bf16(off, MINUS_136, MINUS_136, MINUS_136, MINUS_136, xw[2 * (w & 1)], xw[2 * (w & 1) + 1], zero);
          else mma_bf16(off, MINUS_136, MINUS_136, MINUS_136, MINUS_136, xw[2 * (w & 1)], xw[2 * (w & 1) + 1], off);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          float d[4] = {off[0], off[1], off[2], off[3]};
          const uint32_t* c = &cw[m].x;
#pragma unroll
          for (int w = w0; w < w0 + STEPS; ++w) {
            const uint32_t* xw = &xv[n][w >> 1].x;
            mma_bf16(d, two(c[w], 0), two(c[w], 1), two(c[w], 2), two(c[w], 3), xw[2 * (w & 1)], xw[2 * (w & 1) + 1], d);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[m][n][i] = fmaf(sc[m][i >> 1], d[i], acc[m][n][i]);
        }
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) s_sum[warp][m * TN + g + 8 * (i >> 1)][n * 8 + 2 * t + (i & 1)] = acc[m][n][i];
  __syncthreads();
  for (int e = threadIdx.x; e < MT * TN * M; e += MV_WARPS * 32) {
    const int row = e / (MT * TN), c = e - row * (MT * TN);
    if (n0 + c >= N) continue;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < MV_WARPS; ++w) sum += s_sum[w][c][row];
    y[(size_t)row * N + n0 + c] = __float2bfloat16_rn(sum);
  }
}

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

bool shape_ok(int K, int N, int group) {
  return K >= TK && K % TK == 0 && N >= 1 && (group == 32 || group == 64 || group == 128) && K % group == 0;
}

template <int MT>
void launch(const void* x, const void* codes, const void* scale, int M, int K, int N, int group, void* y,
            cudaStream_t s) {
  const unsigned grid = (unsigned)(((long long)N + MT * TN - 1) / (MT * TN));
  auto go = [&](auto kernel) {
    kernel<<<grid, MV_WARPS * 32, 0, s>>>(static_cast<const uint4*>(x), static_cast<const uint4*>(codes),
                                          static_cast<const __nv_bfloat16*>(scale), M, K, N,
                                          group == 32 ? 5 : (group == 64 ? 6 : 7), static_cast<__nv_bfloat16*>(y));
  };
  if (M <= 8) {
    if (group == 32) go(k_w4_matvec<MT, 1, 2>);
    else go(k_w4_matvec<MT, 1, 4>);
  } else {
    if (group == 32) go(k_w4_matvec<MT, 2, 2>);
    else go(k_w4_matvec<MT, 2, 4>);
  }
}

}  // namespace

extern "C" size_t fc_w4_codes_bytes(int K, int N) {
  if (K < TK || K % TK || N < 1) return 0;
  return (size_t)((N + (long long)TN - 1) / TN) * (K / TK) * TILE_BYTES;
}

extern "C" fc_status fc_w4_pack(const void* d_w, int K, int N, int group, void* d_codes, void* d_scale,
                                fc_stream stream) {
  FC_NVTX_RANGE();
  if (K < 1 || N < 1) return FC_ERR_INVALID_ARG;
  if (!shape_ok(K, N, group)) return FC_ERR_UNSUPPORTED;
  if (!d_w || !d_codes || !d_scale || !aligned(d_w, 16) || !aligned(d_codes, 16) || !aligned(d_scale, 16))
    return FC_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const size_t items = (size_t)(K / group) * N;
  k_w4_scale<<<(unsigned)std::min<size_t>((items + 255) / 256, 152 * 16), 256, 0, s>>>(
      static_cast<const uint16_t*>(d_w), K, N, group, static_cast<__nv_bfloat16*>(d_scale));
  const size_t tiles = (size_t)((N + (long long)TN - 1) / TN) * (K / TK);
  k_w4_pack<<<(unsigned)std::min<size_t>((tiles + 7) / 8, 152 * 16), 256, 0, s>>>(
      static_cast<const __nv_bfloat16*>(d_w), K, N, group, static_cast<const __nv_bfloat16*>(d_scale),
      static_cast<uint4*>(d_codes));
  return FC_CHECK_LAUNCH();
}

extern "C" fc_status fc_w4_matvec(const void* d_x, const void* d_codes, const void* d_scale, int M, int K, int N,
                                  int group, void* d_y, fc_stream stream) {
  FC_NVTX_RANGE();
  if (M < 0 || K < 1 || N < 1) return FC_ERR_INVALID_ARG;
  if (M > 16 || !shape_ok(K, N, group)) return FC_ERR_UNSUPPORTED;
  if (M == 0) return FC_OK;
  if (!d_x || !d_codes || !d_scale || !d_y || !aligned(d_x, 16) || !aligned(d_codes, 16) || !aligned(d_scale, 2) ||
      !aligned(d_y, 2))
    return FC_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (N <= 152 * TN) launch<1>(d_x, d_codes, d_scale, M, K, N, group, d_y, s);
  else launch<2>(d_x, d_codes, d_scale, M, K, N, group, d_y, s);
  return FC_CHECK_LAUNCH();
}
