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
#include <atomic>

#include "fc_common.cuh"

namespace {

constexpr int TK = 64;           // k a tile
constexpr int TN = 16;           // columns a tile
constexpr int TILE_BYTES = 512;
constexpr int MAX_WARPS = 8;     // a CTA
constexpr int FILL = 152 * 8;    // warps that keep HBM busy

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
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Two numbers of a packed word as bf16, exactly: 0x4300 | c is 128 + c, that is
// 136 more than the number.
__device__ __forceinline__ uint32_t two(uint32_t w, int i) {
  uint32_t r;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u), "r"(0x43084308u));
  return r;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory");
}
// The weights' read is the floor: 4.1 to 4.5 bits a weight, each used once.
// Next to it a word's 8 numbers take 7 instructions of the integer pipe and 4
// packed subtractions to become operands.  So the loop's addresses are pointers
// that advance, its stages unrolled, and rows and tiles past the end are read
// from valid places instead of being tested for.
// The operands are the numbers themselves: leaving the 128 + 8 in them and
// taking 136 times the sum of x off again by products of its own cost twenty
// times and more the rounding of these sums, overflowed from x = 2^115 on, and
// took 47 us where this takes 45 (16 x 8192 x 28672; 14.3 and 13.4 for 1 x 8192
// x 8192).
// A warp takes MT tiles of columns (which share the rows of x that it loads)
// and every ks-th tile of k, three in flight by asynchronous copies, x
// AHEAD tiles ahead in registers; with ks = 1 a sum never leaves its warp, else
// the ks warps' sums meet in shared memory.  NT: 8-row tiles of x.  STEPS:
// k-steps that share a scale (the group, or the whole tile).
// At earlier steps of this kernel x four tiles ahead instead of two took 64
// more registers with 16 rows (12 x 8192 x 8192 22.6 us, not 18.5), and seven
// tiles in flight instead of three as long for large weights and a microsecond
// more for small ones.
// Measured: 16 x 8192 x 28672 45 us (126 MB, 2.8 TB/s), a row of it 35 us (3.5
// TB/s), of 2048 x 32256 14 us; 2048 x 2048 5 us a call, 3.5 in a graph.
constexpr int STAGES = 4;
// codes of MT tiles, then the scales [group][MT * TN]
__host__ __device__ constexpr int stage_bytes(int MT, int STEPS) { return MT * TILE_BYTES + MT * TN * 2 * (4 / STEPS); }

template <int MT, int NT, int STEPS>
__global__ void __launch_bounds__(MAX_WARPS * 32) k_w4_matvec(const uint4* __restrict__ x, const uint4* __restrict__ codes,
                                                              const uint16_t* __restrict__ scale, int M, int K, int N,
                                                              int gshift, int ks, __nv_bfloat16* __restrict__ y) {
  extern __shared__ __align__(16) unsigned char smem[];  // rings; then the sums
  constexpr int GROUPS = 4 / STEPS, OFF_SC = MT * TILE_BYTES, STAGE_BYTES = stage_bytes(MT, STEPS);
  constexpr int AHEAD = 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, warps = blockDim.x >> 5;
  const int kt = K / TK, part = warp % ks, tile0 = (blockIdx.x * (warps / ks) + warp / ks) * MT;
  const int n_tiles = (N + TN - 1) / TN;
  const uint32_t ring = smem_u32(smem) + warp * (STAGES * STAGE_BYTES);
  const unsigned char* ring_p = smem + warp * (STAGES * STAGE_BYTES);
  const int n_it = tile0 < n_tiles && part < kt ? (kt - part + ks - 1) / ks : 0;
  // ---- what a step fetches: this lane's part of MT tiles and of their scales
  const uint4* src[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) src[m] = codes + ((size_t)min(tile0 + m, n_tiles - 1) * kt + part) * 32 + lane;
  // two columns' scales of group sq; with MT = 4 a lane has the same of every group
  constexpr int SC_LANES = 8 * MT, SC_EACH = SC_LANES * GROUPS > 32 ? GROUPS : 1;
  const int sq = lane / SC_LANES, sc_c = 2 * (lane % SC_LANES), sc_col = tile0 * TN + sc_c;
  const bool sc_lane = lane < SC_LANES * GROUPS && sc_col < N;
  const uint32_t sc_dst = ring + OFF_SC + (sq * MT * TN + sc_c) * 2;
  const uint16_t* sc_src = scale + sc_col;
  uint32_t sc_k = part * TK + sq * STEPS * 16;
  int to_fetch = n_it;
  auto issue = [&](int stage) {
    if (to_fetch > 0) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        cp_async16(ring + stage * STAGE_BYTES + m * TILE_BYTES + lane * 16, src[m]);
        src[m] += ks * 32;
      }
      if (sc_lane) {
#pragma unroll
        for (int e = 0; e < SC_EACH; ++e) {
          const uint16_t* sp = sc_src + (uint64_t)((sc_k + e * STEPS * 16) >> gshift) * (uint32_t)N;
          const uint32_t dst = sc_dst + stage * STAGE_BYTES + e * MT * TN * 2;
          if (N & 1) {  // rows of odd length: two columns are not one aligned word
            const uint32_t lo = sp[0], hi = sc_col + 1 < N ? sp[1] : 0u;
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(dst), "r"(lo | (hi << 16)) : "memory");
          } else {
            cp_async4(dst, sp);
          }
        }
      }
      sc_k += ks * TK;
      --to_fetch;
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < STAGES - 1; ++i) issue(i);
  // ---- x: rows past M repeat row 0 (their sums are not stored); past the end the last tile is read again
  const uint4* xp[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) xp[n] = x + ((size_t)(n * 8 + g < M ? n * 8 + g : 0) * K + part * TK) / 8 + t;
  int x_left = n_it;
  uint4 xv[AHEAD][NT][2];
  auto load_x = [&](uint4 (&v)[NT][2]) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      v[n][0] = xp[n][0];
      v[n][1] = xp[n][4];
    }
    const int step = --x_left > 0 ? ks * (TK / 8) : 0;
#pragma unroll
    for (int n = 0; n < NT; ++n) xp[n] += step;
  };
  float acc[MT][NT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.f;
  if (n_it > 0) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load_x(xv[i]);
  }
  auto step = [&](int stage, uint4 (&xr)[NT][2]) {
    uint4 cw[MT];
    cp_async_wait<STAGES - 2>();
    __syncwarp();
    const unsigned char* st = ring_p + stage * STAGE_BYTES;
#pragma unroll
    for (int m = 0; m < MT; ++m) cw[m] = *reinterpret_cast<const uint4*>(st + m * TILE_BYTES + lane * 16);
    uint32_t sc[MT][GROUPS][2];
    const uint16_t* sp = reinterpret_cast<const uint16_t*>(st + OFF_SC) + g;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int q = 0; q < GROUPS; ++q)
#pragma unroll
        for (int i = 0; i < 2; ++i) sc[m][q][i] = sp[q * MT * TN + m * TN + 8 * i];
    issue((stage + STAGES - 1) % STAGES);
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) {
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        float d[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) d[n][0] = d[n][1] = d[n][2] = d[n][3] = 0.f;
        const uint32_t* c = &cw[m].x;
#pragma unroll
        for (int w = q * STEPS; w < (q + 1) * STEPS; ++w) {
          const uint32_t c0 = two(c[w], 0), c1 = two(c[w], 1), c2 = two(c[w], 2), c3 = two(c[w], 3);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const uint32_t* xw = &xr[n][w >> 1].x;
            mma_bf16(d[n], c0, c1, c2, c3, xw[2 * (w & 1)], xw[2 * (w & 1) + 1]);
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            acc[m][n][i] = fmaf(__uint_as_float(sc[m][q][i >> 1] << 16), d[n][i], acc[m][n][i]);
      }
    }
    load_x(xr);
  };
#pragma unroll 1
  for (int it = 0; it < n_it; it += STAGES) {
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
      if (it + i >= n_it) break;
      step(i, xv[i % AHEAD]);
    }
  }
  cp_async_wait<0>();
  if (ks == 1) {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int row = n * 8 + 2 * t + (i & 1), col = (tile0 + m) * TN + g + 8 * (i >> 1);
          if (row < M && col < N) y[(size_t)row * N + col] = __float2bfloat16_rn(acc[m][n][i]);
        }
    return;
  }
  __syncthreads();  // every warp is done with its ring
  constexpr int PITCH = NT * 8 + 1;
  float* sums = reinterpret_cast<float*>(smem);  // [warps][MT * TN][PITCH]
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sums[(warp * (MT * TN) + m * TN + g + 8 * (i >> 1)) * PITCH + n * 8 + 2 * t + (i & 1)] = acc[m][n][i];
  __syncthreads();
  const int cols = (warps / ks) * MT * TN, n0 = blockIdx.x * cols;
#pragma unroll 1
  for (int e = threadIdx.x; e < cols * M; e += blockDim.x) {
    const int row = e / cols, c = e - row * cols;
    if (n0 + c >= N) continue;
    const int w0 = c / (MT * TN) * ks, cc = c % (MT * TN);
    float sum = 0.f;
    for (int w = 0; w < ks; ++w) sum += sums[((w0 + w) * (MT * TN) + cc) * PITCH + row];
    y[(size_t)row * N + n0 + c] = __float2bfloat16_rn(sum);
  }
}

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

bool shape_ok(int K, int N, int group) {
  return K >= TK && K % TK == 0 && N >= 1 && (group == 32 || group == 64 || group == 128) && K % group == 0;
}

template <int MT, int NT, int STEPS>
fc_status launch(const void* x, const void* codes, const void* scale, int M, int K, int N, int gshift, void* y,
                 cudaStream_t s) {
  constexpr size_t RING = (size_t)STAGES * stage_bytes(MT, STEPS);           // a warp
  constexpr size_t SUMS = (size_t)MT * TN * (NT * 8 + 1) * sizeof(float);
  constexpr size_t SMEM = RING > SUMS ? RING : SUMS;
  static std::atomic<unsigned long long> done{0};
  const fc_status st = fc_once_per_device(done, [](int) {
    return fc_cuda_status(cudaFuncSetAttribute(k_w4_matvec<MT, NT, STEPS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)(MAX_WARPS * SMEM)));
  });
  if (st != FC_OK) return st;
  // Warps enough for the GPU (FILL): split k while column tiles alone are too
  // few and every part keeps two tiles.
  const int tasks = (int)(((long long)N + MT * TN - 1) / (MT * TN)), kt = K / TK;
  int ks = 1;
  while (ks < MAX_WARPS && (long long)tasks * ks < FILL && kt >= 4 * ks) ks *= 2;
  const int warps = std::max(ks, 4), per = warps / ks;  // small CTAs: they spread over the SMs evenly
  k_w4_matvec<MT, NT, STEPS><<<(unsigned)((tasks + per - 1) / per), warps * 32, warps * SMEM, s>>>(
      static_cast<const uint4*>(x), static_cast<const uint4*>(codes), static_cast<const uint16_t*>(scale), M, K, N,
      gshift, ks, static_cast<__nv_bfloat16*>(y));
  return FC_CHECK_LAUNCH();
}

template <int MT>
fc_status launch_eight(const void* x, const void* codes, const void* scale, int M, int K, int N, int group, void* y,
                       cudaStream_t s) {
  const int gshift = group == 32 ? 5 : (group == 64 ? 6 : 7);
  return group == 32 ? launch<MT, 1, 2>(x, codes, scale, M, K, N, gshift, y, s)
                     : launch<MT, 1, 4>(x, codes, scale, M, K, N, gshift, y, s);
}

template <int MT>
fc_status launch_rows(const void* x, const void* codes, const void* scale, int M, int K, int N, int group, void* y,
                      cudaStream_t s) {
  const int gshift = group == 32 ? 5 : (group == 64 ? 6 : 7);
  if (M <= 8) return launch_eight<MT>(x, codes, scale, M, K, N, group, y, s);
  return group == 32 ? launch<MT, 2, 2>(x, codes, scale, M, K, N, gshift, y, s)
                     : launch<MT, 2, 4>(x, codes, scale, M, K, N, gshift, y, s);
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
  if (!d_x || !d_codes || !d_scale || !d_y || !aligned(d_x, 16) || !aligned(d_codes, 16) || !aligned(d_scale, 16) ||
      !aligned(d_y, 2))
    return FC_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // More column tiles a warp share what it loads of x and what a step costs
  // besides its numbers, fewer fill the GPU sooner (us, replayed from a graph).
  // Two against one: 1 x 8192 x 8192 13.4 instead of 16.1, but 1 x 2048 x 2048
  // 3.8 instead of 3.5, 16 rows of it 4.7 instead of 4.0.  Four against two, up to
  // 8 rows: 8 x 4096 x 20001 24 instead of 31, 1 x 16384 x 32768 81 instead of 83,
  // but 1 x 2048 x 32256 14.1 instead of 13.4 and 8 x 4096 x 11008 13.7 instead of
  // 11.3; 16 rows' sums took too many registers (16 x 8192 x 28672 56 instead of 47
  // when it took that).
  if (N <= 152 * TN * 2) return launch_rows<1>(d_x, d_codes, d_scale, M, K, N, group, d_y, s);
  if (M <= 8 && N > 152 * TN * 8) return launch_eight<4>(d_x, d_codes, d_scale, M, K, N, group, d_y, s);
  return launch_rows<2>(d_x, d_codes, d_scale, M, K, N, group, d_y, s);
}
