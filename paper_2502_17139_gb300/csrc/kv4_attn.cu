// fc_kv4_attn: verification attention over the paged 4-bit cache.
#include <algorithm>
#include <cmath>

#include "fc_common.cuh"
#include "kv4.cuh"

FC_DEFINE_ERROR_WORD(kv4_attn)

namespace {

constexpr int HD = KV4_D;

// ---------------------------------------------------------------------------
// Few query rows for a kv head (n_pad * H / Hkv <= 16: single tokens, small
// trees).  The cache's read bounds this, so the work is what it costs to turn
// 4-bit numbers into tensor-core operands as fast as they arrive.
//
// Keys and dimensions are the rows of mma.m16n8k16 (operand A, from the
// cache), query rows its 8 columns:
//   S^T [16 keys][8 rows] = K Q^T,   O^T [128 dims][8 rows] += V^T P^T.
// fp16 operands: a number c + 8 in a 16-bit half's low bits IS the fp16
// subnormal (c + 8) 2^-24, in the next four bits (c + 8) 2^-20, so a mask is
// all that a pair needs, and a shift every second.  The products are exact.
//   * The 8 too much comes off S in the accumulators' start (-8 times the sum
//     of the query), V by an addition a pair: off O by a second product it
//     would leave errors of a large weight's size on dimensions where that
//     key holds 0.
//   * Queries enter as fp16 times one power of two for the unit (its largest
//     query value below 2^15) and, for the odd dimensions, 1/16.
//   * The second product takes w = 2^(z - m) * (value scale) in fp16.  The
//     row's reference m (O and the row sum are relative to it) moves when a w
//     passes 2^15, to where the largest is 2^11 to 2^12: a running maximum of
//     z + log2(value scale), moved lazily.  (High in fp16's range, so that a
//     weight of 2^-25 of the largest keeps 11 bits.)  For the
//     reference a value scale counts as at least 2^-80, so that 2^(z - m), and
//     the row sum, stay in fp32's range where a row of V is all zeros.  The
//     test for the move is that w is NOT below 2^15: far above the reference
//     2^(z - m) is infinite and its product with a scale of 0 NaN.
// A warp takes every FEW_WARPS-th step of 32 keys (4224 bytes, two runs of 16
// rows in a page), three steps in flight by 16-byte asynchronous copies.  S^T
// becomes P^T's operand by 8x8 transposes in registers.
//
// Key 4g + i of a step (g = lane / 4) is row g of 8-row group i; groups 0, 1
// and 2, 3 make the two products of 16 keys, so that a lane's scales are four
// in a row.  Dimensions 32t .. 32t + 31 (t = lane % 4) are the lane's part of
// K, 16g .. 16g + 15 its part of V, each as they lie in memory; the queries
// are permuted to match.
//
// 32 single tokens over 16384 keys (8 kv heads of 4 query heads, 554 MB) take
// 106 us, 5.2 TB/s: 6.4 TB/s once all run, and some 15 us until they do and
// until the last part is joined.  One token over 131071 keys (138 MB): 37 us.
// There start, end and the instructions (450 a step of a warp, most to place
// numbers) count more than the read.  500 keys: 10 us, latency.
// ---------------------------------------------------------------------------
constexpr int FEW_WARPS = 8, FEW_THREADS = FEW_WARPS * 32;
constexpr int STEP = 32;         // keys a step
constexpr int FEW_STAGES = 3;    // steps in flight a warp
constexpr int OFF_VROWS = STEP * KV4_ROW, OFF_KSC = 2 * STEP * KV4_ROW, OFF_VSC = OFF_KSC + STEP * 2;
constexpr int STEP_BYTES = OFF_VSC + STEP * 2;
// A unit's start and end take a CTA about 6 us, 0.2 us a step at full
// bandwidth; joining two parts of a unit about 4 us.  Parts of 8 steps: 1 x 2000
// and 2 x 1000 keys take 10.3 us where parts of 16 take 12.3, 4 x 4000 14.5 for
// 16.4, but some ragged ones longer (3 requests of up to 3000 keys 13.8 for 12.4,
// 32 of up to 500 11.1 for 10.4); a unit of fewer than CUT_STEPS stays whole (16 x
// 500 keys 10.3 us, in two parts 12.4).
constexpr int UNIT_COST = 30, PART_STEPS = 8, CUT_STEPS = 24;
constexpr float W_MAX = 32768.f;
constexpr int VS_MIN_EXP = -80;
constexpr float VS_MIN = 0x1p-80f;
// A reference before any key: 2^(z + 1e30) is infinite and not below W_MAX
// whatever it is multiplied by, 2^(-1e30 - m) is 0.
constexpr float M_START = -1e30f;

template <int NT>
struct FewSmem {
  static constexpr int ROWS = 8 * NT;
  static constexpr int RING = FEW_WARPS * FEW_STAGES * STEP_BYTES;
  static constexpr int OUT_PITCH = HD + 4;  // floats a row of a warp's partial
  static constexpr int MERGE = FEW_WARPS * ROWS * (OUT_PITCH + 2) * 4;
  static constexpr int JOIN = (ROWS * 152 * 2 + FEW_THREADS * 4) * 4;  // pieces' weights, subsets' sums
  // the new tokens' keys, values and masks (a row of 256 bytes at 272, so that
  // eight rows' reads fall in different banks)
  static constexpr int NEW_PITCH = HD * 2 + 16, NEW = 2 * 16 * NEW_PITCH + 16 * 8;
  static constexpr int OFF_NEW = RING > MERGE ? (RING > JOIN ? RING : JOIN) : (MERGE > JOIN ? MERGE : JOIN);
  static constexpr int BYTES = OFF_NEW + NEW;
};

struct FewArgs {
  Kv4Args a;
  int split;         // 1: units are cut anywhere, by steps; 0: a CTA takes whole units
  uint32_t by_G;     // r / G is r * by_G >> 16 for r < 16
  int* cnt;          // [grid] arrivals at the cut unit that begins in a CTA (at most one does), zero between calls
  float* part;       // [grid][2][ROWS][HD + 2]: O unnormalised, m, l of a CTA's first and last piece
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory");
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// The sum of two fp16 pairs (subnormals kept).
__device__ __forceinline__ uint32_t less8(uint32_t v, uint32_t minus) {
  uint32_t r;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(minus));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ int expo(float x) { return (int)((__float_as_uint(x) >> 23) & 255u) - 127; }
__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// A staged step keeps row r's 16-byte chunk c at
//   (r % 4 + 4 (r / 8)) * 128 + ((r / 4 + r / 8) % 2) * 64 + (c ^ 2 (r / 16)) * 16:
// two rows a 128-byte line, such that a quarter warp's 16-byte reads (rows 8x
// + i and 8x + 4 + i) and a half warp's 8-byte reads (rows 8t + i, t = 0..3,
// two chunks) each fall in different banks.  Every address below is one of
// three lane constants plus an immediate.

// steps of a length up to 2^31 - 1, whose rounding up passes an int
__device__ __forceinline__ int steps_of(int kvl) { return (int)(((uint32_t)kvl + STEP - 1) / STEP); }

__device__ __forceinline__ int few_steps(const Kv4Args& a, int b, int& nn, int& kvl, bool& bad) {
  kvl = a.kv_len[b];
  nn = a.n_nodes ? a.n_nodes[b] : a.n_pad;
  bad = nn < 0 || nn > a.n_pad || kvl < 0 || kvl > (long long)a.max_pages << a.shift;
  if (bad) nn = kvl = 0;
  return nn == 0 ? 1 : max(1, steps_of(kvl) + (a.k_new ? 1 : 0));
}

// parts that a unit of so many steps is worth (0: like 1)
__device__ __forceinline__ int parts_of(int steps) { return steps < CUT_STEPS ? 0 : steps / PART_STEPS; }

template <int NT>
__global__ void __launch_bounds__(FEW_THREADS, NT == 1 ? 2 : 1) k_kv4_attn_few(FewArgs f) {
  using L = FewSmem<NT>;
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ int s_last;
  const Kv4Args& a = f.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const uint32_t ring = smem_u32(smem) + warp * (FEW_STAGES * STEP_BYTES);
  const unsigned char* ring_p = smem + warp * (FEW_STAGES * STEP_BYTES);

  // How the units' steps are dealt out, from every request's length (the host
  // has seen to it that the sums fit 32 bits):
  //   even     every unit in the same number of parts, a CTA each: no CTA
  //            works on two units, the longest unit sets the time;
  //   balanced shares of equal cost, cut anywhere, a unit costing its steps
  //            and UNIT_COST for its start and end.
  int cur, end, b = 0, req_base = 0;  // req_base: first cost of request b
  int parts = 0;                      // even: parts a unit; 0: balanced
  const int units = a.B * a.Hkv;
  Kv4Cut cut(1, 1, 1);
  if (f.split) {  // every warp for itself
    int nn, kvl;
    bool bad;
    const int first = lane < a.B ? few_steps(a, lane, nn, kvl, bad) + UNIT_COST : 0;
    int sum = first, longest = first;
#pragma unroll 1
    for (int i = lane + 32; i < a.B; i += 32) {
      const int st = few_steps(a, i, nn, kvl, bad) + UNIT_COST;
      sum += st;
      longest = max(longest, st);
    }
    cut = Kv4Cut(__reduce_add_sync(0xFFFFFFFFu, sum) * a.Hkv, gridDim.x, UNIT_COST + PART_STEPS);
    longest = __reduce_max_sync(0xFFFFFFFFu, longest);
    if (units <= (int)gridDim.x) {
      const int k = max(1, min((int)gridDim.x / units, parts_of(longest - UNIT_COST)));
      if ((longest - UNIT_COST) / k <= cut.q) parts = k;
    }
    if (parts) {
      cur = blockIdx.x;  // a part
      end = min(units * parts, cur + 1);
    } else {
      cur = (int)blockIdx.x < cut.n ? cut.start(blockIdx.x) : 0;
      end = (int)blockIdx.x < cut.n ? cut.start(blockIdx.x + 1) : 0;
#pragma unroll 1
      for (int b0 = 0; b0 < a.B; b0 += 32) {
        const int mine =
            (b0 == 0 ? first : (b0 + lane < a.B ? few_steps(a, b0 + lane, nn, kvl, bad) + UNIT_COST : 0)) * a.Hkv;
        int inc = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xFFFFFFFFu, inc, o);
          if (lane >= o) inc += v;
        }
        const uint32_t hit = __ballot_sync(0xFFFFFFFFu, req_base + inc > cur);
        if (hit) {
          const int w = __ffs(hit) - 1;
          b = b0 + w;
          req_base += __shfl_sync(0xFFFFFFFFu, inc - mine, w);
          break;
        }
        req_base += __shfl_sync(0xFFFFFFFFu, inc, 31);
      }
    }
  } else {
    cur = blockIdx.x;  // a unit
    end = units;
  }

#pragma unroll 1
  while (cur < end) {
    // ---- the next unit, this CTA's steps [s0, s1) of it, and the CTAs [c0, c0 + nc) that share it
    int nn, kvl, gh, s0 = 0, s1, steps, c0 = 0, nc = 1, unit_base = 0;
    bool bad;
    if (f.split && !parts) {
      steps = few_steps(a, b, nn, kvl, bad);
#pragma unroll 1
      while (cur - req_base >= (steps + UNIT_COST) * a.Hkv) {
        req_base += (steps + UNIT_COST) * a.Hkv;
        ++b;
        steps = few_steps(a, b, nn, kvl, bad);
      }
      gh = (cur - req_base) / (steps + UNIT_COST);
      unit_base = req_base + gh * (steps + UNIT_COST);
      s0 = max(0, cur - unit_base - UNIT_COST);
      cur = min(unit_base + UNIT_COST + steps, end);
      s1 = cur - unit_base - UNIT_COST;
      if (s1 <= s0) break;  // the share ends before the unit's first step
      c0 = cut.share_of(unit_base + UNIT_COST);
      nc = cut.share_of(unit_base + UNIT_COST + steps - 1) - c0 + 1;
    } else {
      const int unit = f.split ? cur / parts : cur;
      b = unit / a.Hkv;
      gh = unit - b * a.Hkv;
      steps = few_steps(a, b, nn, kvl, bad);
      s1 = steps;
      cur += gridDim.x;
      if (f.split) {
        c0 = unit * parts;
        nc = max(1, min(parts, parts_of(steps)));  // a short unit in fewer parts
        const int part = (int)blockIdx.x - c0, q = steps / nc, rem = steps - q * nc;
        if (part >= nc) break;
        s0 = part * q + min(part, rem);
        s1 = s0 + q + (part < rem ? 1 : 0);
      }
    }
    // where CTA c keeps its piece of this unit: a balanced share's second piece apart from its first
    auto piece = [&](int c) {
      return f.part + (2 * c + (!parts && cut.start(c) < unit_base ? 1 : 0)) * (L::ROWS * (HD + 2));
    };
    if (bad && gh == 0 && s0 == 0 && tid == 0) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_INVALID);
    const int c_steps = nn == 0 ? 0 : steps_of(kvl);
    const int R = nn * a.G;  // rows in use: node-major, r = node * G + head in group
    auto node_of = [&](int r) { return (int)((uint32_t)r * f.by_G >> 16); };
    auto q_row = [&](int r) {
      const int i = node_of(r);
      return a.q + (((size_t)b * a.n_pad + i) * a.H + gh * a.G + (r - i * a.G)) * HD;
    };

    const uint8_t *k_lane = a.kc + lane * 16, *v_lane = a.vc + lane * 16;
    const __nv_bfloat16* sc0 = (lane & 4) ? a.vs : a.ks;
    const uint8_t* sc_lane = reinterpret_cast<const uint8_t*>(sc0) + (lane & 1) * 16;
    const uint32_t put0 = ring + ((lane >> 2) & 3) * 128 + (lane >> 4) * 64 + (lane & 3) * 16;
    const int get_k = (g >> 1) * 512 + ((g ^ (g >> 1)) & 1) * 64 + ((t ^ ((g >> 2) << 1)) << 4);
    const int get_v = OFF_VROWS + t * 512 + (t & 1) * 64 + (((g >> 1) ^ ((t >> 1) << 1)) << 4) + (g & 1) * 8;
    // ---- cached steps of this warp: s0 + warp, s0 + warp + 8, ...
    const int cs1 = min(s1, c_steps);
    const int n_it = cs1 > s0 + warp ? (cs1 - s0 - warp + FEW_WARPS - 1) / FEW_WARPS : 0;
    int id_a = 0, id_b = 0;  // page ids of the two runs of 16 keys of the warp's next 32 steps, one a lane
    uint32_t outside = 0;    // bits 2 x stage, + 1: that run's page is not in the pool
    const int32_t* tab = a.table + (size_t)b * a.max_pages;
    // runs of 16 rows are counted in 32 bits (1024 bytes each: 4 TB)
    const uint32_t runs_page = (uint32_t)a.Hkv << (a.shift - 4), run0 = (uint32_t)gh << (a.shift - 4);
    const uint32_t run_mask = (1u << (a.shift - 4)) - 1u;
    auto issue = [&](int it, int stage, uint32_t at) {
      if (it < n_it) {
        const int s = s0 + warp + it * FEW_WARPS;
        if ((it & 31) == 0) {
          const long long key = (long long)(s + lane * FEW_WARPS) * STEP;
          id_a = key < kvl ? tab[key >> a.shift] : 0;
          id_b = a.shift == 4 && key + 16 < kvl ? tab[(key + 16) >> 4] : 0;
        }
        int ia = __shfl_sync(0xFFFFFFFFu, id_a, it & 31);
        uint32_t ra, rb;
        if (a.shift > 4) {  // both runs in one page
          if ((unsigned)ia >= (unsigned)a.n_pages) {  // its keys are left out below
            outside |= 3u << (2 * stage);
            ia = 0;
          }
          ra = ia * runs_page + (run0 + ((uint32_t)(2 * s) & run_mask));
          rb = ra + 1;
        } else {
          int ib = __shfl_sync(0xFFFFFFFFu, id_b, it & 31);
          if (max((unsigned)ia, (unsigned)ib) >= (unsigned)a.n_pages) {
            const bool xa = (unsigned)ia >= (unsigned)a.n_pages, xb = (unsigned)ib >= (unsigned)a.n_pages;
            outside |= ((xa ? 1u : 0u) | (xb ? 2u : 0u)) << (2 * stage);
            ia = xa ? 0 : ia;
            ib = xb ? 0 : ib;
          }
          ra = ia * runs_page + run0;
          rb = ib * runs_page + run0;
        }
        const uint32_t d0 = put0 + at, d1 = d0 ^ 64u, d2 = d0 ^ 32u, d3 = d0 ^ 96u;
        const uint8_t *ka = k_lane + (uint64_t)ra * 1024u, *kb = k_lane + (uint64_t)rb * 1024u;
        const uint8_t *va = v_lane + (uint64_t)ra * 1024u, *vb = v_lane + (uint64_t)rb * 1024u;
        cp_async16(d0, ka);
        cp_async16(d1 + 512, ka + 512);
        cp_async16(d2 + 1024, kb);
        cp_async16(d3 + 1536, kb + 512);
        cp_async16(d0 + OFF_VROWS, va);
        cp_async16(d1 + OFF_VROWS + 512, va + 512);
        cp_async16(d2 + OFF_VROWS + 1024, vb);
        cp_async16(d3 + OFF_VROWS + 1536, vb + 512);
        if (lane < 8)  // K scales of the two runs, then V scales
          cp_async16(ring + at + OFF_KSC + lane * 16, sc_lane + (uint64_t)((lane & 2) ? rb : ra) * 32u);
      }
      cp_async_commit();
    };
    // ---- queries: the unit's power of two, then the operand registers
    // k-step 2i of word i of a key's 16-byte quarter t: dimensions 32t + 8i +
    // {0, 4} and {1, 5} / 16; k-step 2i + 1: {2, 6} and {3, 7} / 16
    uint4 qw[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        qw[n][i] = 8 * n + g < R ? reinterpret_cast<const uint4*>(q_row(8 * n + g))[4 * t + i] : make_uint4(0, 0, 0, 0);
    // the new tokens' rows and masks, by the warp that will use them
    auto new_here = [&] { return a.k_new && nn > 0 && s1 == steps && warp == (steps - 1 - s0) % FEW_WARPS; };
    if (new_here()) {
      const uint32_t to = smem_u32(smem) + L::OFF_NEW;
      const size_t from = ((size_t)b * a.Hkv + gh) * a.n_pad * HD + (lane & 15) * 8;
#pragma unroll 1
      for (int j = lane >> 4; j < nn; j += 2) {
        cp_async16(to + j * L::NEW_PITCH + (lane & 15) * 16, a.k_new + from + (size_t)j * HD);
        cp_async16(to + (16 + j) * L::NEW_PITCH + (lane & 15) * 16, a.v_new + from + (size_t)j * HD);
      }
      if (a.mask && lane < nn) cp_async8(to + 32 * L::NEW_PITCH + lane * 8, a.mask + (size_t)b * a.n_pad + lane);
    }
    // the first steps are asked for before the queries have come
#pragma unroll 1
    for (int it = 0; it < FEW_STAGES - 1; ++it) issue(it, it, it * STEP_BYTES);
    uint32_t top = 0;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t* w = &qw[n][i].x;
#pragma unroll
        for (int x = 0; x < 4; ++x) {  // magnitudes of finite values, both halves at once
          const uint32_t mag = w[x] & 0x7FFF7FFFu;
          top = __vmaxu2(top, mag & ~__vcmpgeu2(mag, 0x7F807F80u));
        }
      }
    top = __reduce_max_sync(0xFFFFFFFFu, max(top & 0xFFFFu, top >> 16));
    const int qe = top ? min(max((int)(top >> 7) - 127, -100), 100) : 0;  // largest |q| < 2^(qe + 1) (or it overflows)
    const float q_mul = pow2i(14 - qe), q_odd = q_mul * 0.0625f;
    const float z_mul = a.scale_log2 * pow2i(qe + 10);  // undoes 2^(14 - qe) 2^-24
    uint32_t qf[NT][8][2];
    float s_init[NT][2];  // rows 8n + 2t, + 1: -8 2^-24 times the sum of the row
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 w = qw[n][i];
        const float d0 = lo_f(w.x) * q_mul, d1 = hi_f(w.x) * q_odd, d2 = lo_f(w.y) * q_mul, d3 = hi_f(w.y) * q_odd;
        const float d4 = lo_f(w.z) * q_mul, d5 = hi_f(w.z) * q_odd, d6 = lo_f(w.w) * q_mul, d7 = hi_f(w.w) * q_odd;
        qf[n][2 * i][0] = pack_f16x2(d0, d4);
        qf[n][2 * i][1] = pack_f16x2(d1, d5);
        qf[n][2 * i + 1][0] = pack_f16x2(d2, d6);
        qf[n][2 * i + 1][1] = pack_f16x2(d3, d7);
        sum += ((d0 + d2) + (d4 + d6)) + 16.f * ((d1 + d3) + (d5 + d7));
      }
      sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
      sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);  // row g of the tile, in all four lanes t
      sum *= -0x1p-21f;
      s_init[n][0] = __shfl_sync(0xFFFFFFFFu, sum, 8 * t);      // row 2t is lane group g = 2t
      s_init[n][1] = __shfl_sync(0xFFFFFFFFu, sum, 8 * t + 4);
    }

    float o[NT][8][4];  // [tile of 16 dims][c]: rows 2t + (c & 1), dims 16g + 2 mt + (c >> 1)
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int mt = 0; mt < 8; ++mt)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[n][mt][c] = 0.f;
      m[n][0] = m[n][1] = M_START;
      l[n][0] = l[n][1] = 0.f;
    }

    // Scores d * ks (base 2; masked keys: d -inf, ks 1; d[i][r] of the lane's
    // key i, row 2t + r) and value scales to w = 2^(d ks - m) vs; adds the
    // powers to the row sums; moves the references when a w is too large.  A
    // NaN of one row's moves the other's for nothing, which harms no result.
    auto weigh = [&](int n, const float (&d)[4][2], const float (&ks)[4], const float (&vs)[4], float (&w)[4][2]) {
      float p[4][2];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          p[i][r] = exp2_fast(fmaf(d[i][r], ks[i], -m[n][r]));
          w[i][r] = p[i][r] * vs[i];
        }
      float ps[2] = {(p[0][0] + p[1][0]) + (p[2][0] + p[3][0]), (p[0][1] + p[1][1]) + (p[2][1] + p[3][1])};
      const float sum = ((w[0][0] + w[0][1]) + (w[1][0] + w[1][1])) + ((w[2][0] + w[2][1]) + (w[3][0] + w[3][1]));
      if (__any_sync(0xFFFFFFFFu, !(fmaf(ps[0] + ps[1], VS_MIN, sum) <= W_MAX))) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float top = M_START;
#pragma unroll
          for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaf(d[i][r], ks[i], (float)(max(expo(vs[i]), VS_MIN_EXP) - 11)));
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
          const float mn = fmaxf(m[n][r], top), al = exp2_fast(m[n][r] - mn);
          m[n][r] = mn;
          l[n][r] *= al;
#pragma unroll
          for (int mt = 0; mt < 8; ++mt) o[n][mt][r] *= al, o[n][mt][2 + r] *= al;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            p[i][r] = exp2_fast(fmaf(d[i][r], ks[i], -mn));
            w[i][r] = p[i][r] * vs[i];
          }
          ps[r] = (p[0][r] + p[1][r]) + (p[2][r] + p[3][r]);
        }
      }
      l[n][0] += ps[0];
      l[n][1] += ps[1];
    };

    // ---- the loop over the steps
    int stage = 0;
    for (int it = 0; it < n_it; ++it) {
      cp_async_wait<FEW_STAGES - 2>();
      __syncwarp();
      const unsigned char* st = ring_p + stage * STEP_BYTES;
      const int left = kvl - (s0 + warp + it * FEW_WARPS) * STEP;  // keys of the request from here on
      const uint32_t out_now = (outside >> (2 * stage)) & 3u;
      outside &= ~(3u << (2 * stage));
      {  // into the stage read in the last turn
        const int last = stage == 0 ? FEW_STAGES - 1 : stage - 1;
        issue(it + FEW_STAGES - 1, last, last * STEP_BYTES);
      }
      const uint2 ks2 = *reinterpret_cast<const uint2*>(st + OFF_KSC + 8 * g);
      const uint2 vs2 = *reinterpret_cast<const uint2*>(st + OFF_VSC + 8 * g);
      float ks[4] = {lo_f(ks2.x) * z_mul, hi_f(ks2.x) * z_mul, lo_f(ks2.y) * z_mul, hi_f(ks2.y) * z_mul};
      float vs[4] = {lo_f(vs2.x), hi_f(vs2.x), lo_f(vs2.y), hi_f(vs2.y)};
      float z[NT][4][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // keys 4g + 2h, 4g + 2h + 1
        const uint4 k0 = *reinterpret_cast<const uint4*>(st + get_k + h * 256);
        const uint4 k1 = *reinterpret_cast<const uint4*>(st + get_k + h * 256 + 128);
        float d[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) d[n][0] = d[n][2] = s_init[n][0], d[n][1] = d[n][3] = s_init[n][1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = (&k0.x)[i], y = (&k1.x)[i];
          const uint32_t x8 = x >> 8, y8 = y >> 8;
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma_f16(d[n], x & 0x000F000Fu, y & 0x000F000Fu, x & 0x00F000F0u, y & 0x00F000F0u, qf[n][2 * i][0],
                    qf[n][2 * i][1]);
            mma_f16(d[n], x8 & 0x000F000Fu, y8 & 0x000F000Fu, x8 & 0x00F000F0u, y8 & 0x00F000F0u, qf[n][2 * i + 1][0],
                    qf[n][2 * i + 1][1]);
          }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) z[n][2 * h + (c >> 1)][c & 1] = d[n][c];
      }
      if (left < STEP || out_now) {
        if (out_now && lane == 0) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_INVALID);
        // keys past the request's end, or in a page outside the pool: no weight, whatever stands there
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int j = 4 * g + i;
          if (j >= left || ((out_now >> (j >> 4)) & 1u)) {
            vs[i] = 0.f;
            ks[i] = 1.f;
#pragma unroll
            for (int n = 0; n < NT; ++n) z[n][i][0] = z[n][i][1] = -INFINITY;
          }
        }
      }
      uint32_t pb[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float w[4][2];
        weigh(n, z[n], ks, vs, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) pb[n][i] = transpose8x8(pack_f16x2(w[i][0], w[i][1]));
      }
      // O^T: in product h, k 2t, 2t + 1 are rows 2t, 2t + 1 of group 2h (keys
      // 8t + 2h, 8t + 4 + 2h), k 2t + 8, + 9 those of group 2h + 1
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint2 va = *reinterpret_cast<const uint2*>(st + get_v + h * 256);
        const uint2 vb = *reinterpret_cast<const uint2*>(st + (get_v ^ 64) + h * 256);
        const uint2 vc = *reinterpret_cast<const uint2*>(st + get_v + h * 256 + 128);
        const uint2 vd = *reinterpret_cast<const uint2*>(st + (get_v ^ 64) + h * 256 + 128);
#pragma unroll
        for (int u = 0; u < 4; ++u) {  // four dims: a 16-bit part of each key's word
          const uint32_t sel = (u & 1) ? 0x7632u : 0x5410u;
          const uint32_t x = __byte_perm((&va.x)[u >> 1], (&vb.x)[u >> 1], sel);
          const uint32_t y = __byte_perm((&vc.x)[u >> 1], (&vd.x)[u >> 1], sel);
          const uint32_t x8 = x >> 8, y8 = y >> 8;
          const uint32_t v0 = less8(x & 0x000F000Fu, 0x80088008u), v1 = less8(x & 0x00F000F0u, 0x80808080u);
          const uint32_t v2 = less8(y & 0x000F000Fu, 0x80088008u), v3 = less8(y & 0x00F000F0u, 0x80808080u);
          const uint32_t v4 = less8(x8 & 0x000F000Fu, 0x80088008u), v5 = less8(x8 & 0x00F000F0u, 0x80808080u);
          const uint32_t v6 = less8(y8 & 0x000F000Fu, 0x80088008u), v7 = less8(y8 & 0x00F000F0u, 0x80808080u);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma_f16(o[n][2 * u], v0, v1, v2, v3, pb[n][2 * h], pb[n][2 * h + 1]);
            mma_f16(o[n][2 * u + 1], v4, v5, v6, v7, pb[n][2 * h], pb[n][2 * h + 1]);
          }
        }
      }
      stage = stage == FEW_STAGES - 1 ? 0 : stage + 1;
    }
    cp_async_wait<0>();

    // ---- the new tokens' step, in bf16: the warp whose turn it would be
    if (new_here()) {
      __syncwarp();
      const unsigned char* rows = smem + L::OFF_NEW;
      const uint64_t* masks = reinterpret_cast<const uint64_t*>(rows + 32 * L::NEW_PITCH);
      const uint4 zero = make_uint4(0, 0, 0, 0);
      float z[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) z[n][0] = z[n][1] = z[n][2] = z[n][3] = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 x = g < nn ? reinterpret_cast<const uint4*>(rows + g * L::NEW_PITCH)[4 * t + i] : zero;
        const uint4 y = g + 8 < nn ? reinterpret_cast<const uint4*>(rows + (g + 8) * L::NEW_PITCH)[4 * t + i] : zero;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint4 w = 8 * n + g < R ? reinterpret_cast<const uint4*>(q_row(8 * n + g))[4 * t + i] : zero;
          mma_bf16(z[n], x.x, y.x, x.y, y.y, w.x, w.y);
          mma_bf16(z[n], x.z, y.z, x.w, y.w, w.z, w.w);
        }
      }
      uint32_t pb[NT][2], seen = 0, bad = 0;  // bits 4n + c: z[n][c]'s key is seen; bits j: values of token j are not finite
      const float one[4] = {1.f, 1.f, 0.f, 0.f};
      const float by[4] = {a.scale_log2, a.scale_log2, 1.f, 1.f};
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float zz[4][2], w[4][2];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int r = 8 * n + 2 * t + (c & 1), j = g + 8 * (c >> 1), i = node_of(r);
          bool sees = r < R && j < nn;
          if (sees) sees = a.mask ? (masks[i] >> j) & 1 : j <= i;
          seen |= (sees ? 1u : 0u) << (4 * n + c);
          zz[c >> 1][c & 1] = sees ? z[n][c] : -INFINITY;
          zz[2 + (c >> 1)][c & 1] = -INFINITY;
        }
        weigh(n, zz, by, one, w);
        // O is held times 2^-24 (2^-20 at odd dims): the weights take 2^-24, the odd dims' values 16
        pb[n][0] = transpose8x8(pack_bf16x2(w[0][0] * 0x1p-24f, w[0][1] * 0x1p-24f));
        pb[n][1] = transpose8x8(pack_bf16x2(w[1][0] * 0x1p-24f, w[1][1] * 0x1p-24f));
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // 8 of the lane's 16 dims
        uint4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int j = 2 * t + (k & 1) + 8 * (k >> 1);
          v[k] = j < nn ? reinterpret_cast<const uint4*>(rows + (16 + j) * L::NEW_PITCH)[2 * g + h] : zero;
          // a value that is not finite becomes 0, as no weight of 0 would take
          // it out of the rows that do not see its token; those that do are NaN
          uint32_t* w = &v[k].x;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const uint32_t not_finite = __vcmpgeu2(w[u] & 0x7FFF7FFFu, 0x7F807F80u);
            w[u] &= ~not_finite;
            if (not_finite) bad |= 1u << j;
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          auto odd = [](uint32_t w) { return pack_bf16x2(lo_f(w) * 16.f, hi_f(w) * 16.f); };
          const uint32_t a0 = __byte_perm((&v[0].x)[u], (&v[1].x)[u], 0x5410), a1 = odd(__byte_perm((&v[0].x)[u], (&v[1].x)[u], 0x7632));
          const uint32_t a2 = __byte_perm((&v[2].x)[u], (&v[3].x)[u], 0x5410), a3 = odd(__byte_perm((&v[2].x)[u], (&v[3].x)[u], 0x7632));
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_bf16(o[n][4 * h + u], a0, a1, a2, a3, pb[n][0], pb[n][1]);
        }
      }
      bad = __reduce_or_sync(0xFFFFFFFFu, bad);
      if (bad) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (((seen >> (4 * n + c)) & 1u) && ((bad >> (g + 8 * (c >> 1))) & 1u)) l[n][c & 1] = __uint_as_float(0x7FC00000u);
      }
    }

    // ---- join the warps, then the CTAs of a cut unit
    __syncthreads();  // every warp is done with the ring
    float* po = reinterpret_cast<float*>(smem);
    float2* pml = reinterpret_cast<float2*>(po + FEW_WARPS * L::ROWS * L::OUT_PITCH);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float sum = l[n][r];
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
        const int row = warp * L::ROWS + 8 * n + 2 * t + r;
        constexpr float up = 0x1p24f, up_odd = 0x1p20f;
        float* dst = po + row * L::OUT_PITCH + 16 * g;
#pragma unroll
        for (int mt = 0; mt < 8; mt += 2)
          *reinterpret_cast<float4*>(dst + 2 * mt) = make_float4(o[n][mt][r] * up, o[n][mt][2 + r] * up_odd,
                                                                 o[n][mt + 1][r] * up, o[n][mt + 1][2 + r] * up_odd);
        if (g == 0) pml[row] = make_float2(m[n][r], sum);
      }
    __syncthreads();
    const bool whole = s0 == 0 && s1 == steps;
    const int rows_all = a.n_pad * a.G;  // rows past the nodes are written as zeros
    float* slot = piece(blockIdx.x);
    auto put = [&](int r, int d4, const float4& v) {
      const int i = node_of(r);
      __nv_bfloat16* dst = a.out + (((size_t)b * a.n_pad + i) * a.H + gh * a.G + (r - i * a.G)) * HD + 4 * d4;
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
    };
#pragma unroll 1
    for (int e = tid; e < rows_all * (HD / 4); e += FEW_THREADS) {
      const int r = e / (HD / 4), d4 = e % (HD / 4);
      if (r >= R) {
        if (s0 == 0) put(r, d4, make_float4(0.f, 0.f, 0.f, 0.f));
        continue;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int w = 0; w < FEW_WARPS; ++w) mx = fmaxf(mx, pml[w * L::ROWS + r].x);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < FEW_WARPS; ++w) {
        const float2 ml = pml[w * L::ROWS + r];
        const float k = exp2_fast(ml.x - mx);
        const float4 v = *reinterpret_cast<const float4*>(po + (w * L::ROWS + r) * L::OUT_PITCH + 4 * d4);
        sum += ml.y * k;
        acc.x += v.x * k, acc.y += v.y * k, acc.z += v.z * k, acc.w += v.w * k;
      }
      if (whole) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        put(r, d4, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
      } else {
        __stcg(reinterpret_cast<float4*>(slot + r * HD) + d4, acc);
        if (d4 == 0) __stcg(reinterpret_cast<float2*>(slot + L::ROWS * HD) + r, make_float2(mx, sum));
      }
    }
    if (!whole) {
      // The last CTA to arrive adds up the pieces, in CTA order whichever it is.
      __threadfence();
      __syncthreads();
      if (tid == 0) s_last = atomicAdd(f.cnt + c0, 1) == nc - 1;
      __syncthreads();
      if (s_last) {
        __threadfence();
        if (tid == 0) f.cnt[c0] = 0;  // fit for the next call
        // each piece's weight in a row, a warp a row ...
        float* wt = reinterpret_cast<float*>(smem);  // [R][nc]
        float* red = wt + ((R * nc + 3) & ~3);       // [subsets][R][HD]
#pragma unroll 1
        for (int r = warp; r < R; r += FEW_WARPS) {
          float mx = -INFINITY, sum = 0.f;
#pragma unroll 2
          for (int c = lane; c < nc; c += 32) {
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(piece(c0 + c) + L::ROWS * HD) + r);
            const float mn = fmaxf(mx, ml.x);
            sum = sum * exp2_fast(mx - mn) + ml.y * exp2_fast(ml.x - mn);
            mx = mn;
            wt[r * nc + c] = ml.x;
          }
          float all = mx;
#pragma unroll
          for (int x = 16; x > 0; x >>= 1) all = fmaxf(all, __shfl_xor_sync(0xFFFFFFFFu, all, x));
          sum *= exp2_fast(mx - all);
#pragma unroll
          for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll 1
          for (int c = lane; c < nc; c += 32) wt[r * nc + c] = exp2_fast(wt[r * nc + c] - all) * inv;
        }
        __syncthreads();
        // ... then its values, the pieces dealt out to as many subsets as there are threads for
        const int quads = R * (HD / 4), subsets = max(1, FEW_THREADS / quads);
#pragma unroll 1
        for (int e = tid; e < quads * subsets; e += FEW_THREADS) {
          const int sub = e / quads, q = e - sub * quads, r = q / (HD / 4), d4 = q % (HD / 4);
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
          for (int c = sub; c < nc; c += subsets) {
            const float k = wt[r * nc + c];
            const float4 v = __ldcg(reinterpret_cast<const float4*>(piece(c0 + c) + r * HD) + d4);
            acc.x += v.x * k, acc.y += v.y * k, acc.z += v.z * k, acc.w += v.w * k;
          }
          if (subsets == 1) put(r, d4, acc);
          else reinterpret_cast<float4*>(red)[e] = acc;
        }
        if (subsets > 1) {
          __syncthreads();
#pragma unroll 1
          for (int q = tid; q < quads; q += FEW_THREADS) {
            float4 acc = reinterpret_cast<const float4*>(red)[q];
#pragma unroll 1
            for (int sub = 1; sub < subsets; ++sub) {
              const float4 v = reinterpret_cast<const float4*>(red)[sub * quads + q];
              acc.x += v.x, acc.y += v.y, acc.z += v.z, acc.w += v.w;
            }
            put(q / (HD / 4), q % (HD / 4), acc);
          }
        }
      }
    }
    __syncthreads();  // the partials are read; the ring is free again
  }
}

constexpr int FEW_GRID = 152 * 2;

static_assert(FEW_GRID * sizeof(int) <= KV4_WS_COUNTERS, "room for the counters");

template <int NT>
fc_status launch_few(const Kv4Args& a, void* ws, size_t ws_bytes, cudaStream_t s) {
  static std::atomic<unsigned long long> done{0};
  const fc_status st = fc_once_per_device(done, [](int) {
    return fc_cuda_status(cudaFuncSetAttribute(k_kv4_attn_few<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               FewSmem<NT>::BYTES));
  });
  if (st != FC_OK) return st;
  const int full = NT == 1 ? FEW_GRID : FEW_GRID / 2;
  const size_t cnt = KV4_WS_COUNTERS, one = (size_t)2 * FewSmem<NT>::ROWS * (HD + 2) * sizeof(float);
  const long long units = (long long)a.B * a.Hkv;
  // at most what the tables could hold, in steps (past 32 bits there are units enough without cutting them)
  const long long longest = (((long long)a.max_pages << a.shift) + STEP - 1) / STEP + 1, most = units * (longest + UNIT_COST);
  int grid = (int)std::min<long long>(full, units * std::max<long long>(1, longest / PART_STEPS));
  FewArgs f{a, 1, 65536u / a.G + 1, nullptr, nullptr};
  if (ws && ws_bytes > cnt) grid = (int)std::min<size_t>(grid, (ws_bytes - cnt) / one);
  // a workspace for fewer CTAs than whole units would fill: whole units (16 x 8000 keys on two CTAs
  // 1.09 ms, whole units 0.04)
  if (!ws || ws_bytes <= cnt || grid < std::min<long long>(full, units) || most > 0x7FFFFFFFll) {
    f.split = 0;
    grid = (int)std::min<long long>(units, 1 << 20);
  } else {
    f.cnt = static_cast<int*>(ws);
    f.part = reinterpret_cast<float*>(static_cast<unsigned char*>(ws) + cnt);
  }
  k_kv4_attn_few<NT><<<grid, FEW_THREADS, FewSmem<NT>::BYTES, s>>>(f);
  return FC_CHECK_LAUNCH();
}

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

bool shape_ok(int n_pad, int H, int Hkv) {
  return n_pad >= 1 && n_pad <= FC_MAX_NODES && H >= 1 && Hkv >= 1 && H % Hkv == 0 && H / Hkv <= 16;
}

}  // namespace

extern "C" size_t fc_kv4_attn_workspace(int batch, int n_pad, int H, int Hkv) {
  if (batch < 1 || !shape_ok(n_pad, H, Hkv)) return 0;
  const int rows = n_pad * (H / Hkv);
  if (rows > 16) return kv4_attn_many_workspace(batch, n_pad, H, Hkv);
  return KV4_WS_COUNTERS + (size_t)FEW_GRID * 2 * 8 * (HD + 2) * sizeof(float);
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
      !aligned(d_k_new, 16) || !aligned(d_v_new, 16) || !aligned(d_mask, 8) || (d_ws && !aligned(d_ws, 256)))
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
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if ((long long)batch * a.Hkv > 1ll << 30) return FC_ERR_UNSUPPORTED;
  // Measured on both sides of the rules (8 kv heads of 4 query heads):
  //   4 rows, 32 x 16384 keys:  one 8-row tile 106 us, two 154
  //   16 rows, 32 x 8192 keys:  two 8-row tiles 91 us, a tcgen05 tile 174;
  //            1 x 500 keys: 12 and 22
  // (three 8-row tiles would not fit the registers).
  if (n_pad * a.G <= 8) return launch_few<1>(a, d_ws, ws_bytes, s);
  if (n_pad * a.G <= 16) return launch_few<2>(a, d_ws, ws_bytes, s);
  return kv4_attn_many(a, d_ws, ws_bytes, s);
}
