// fc_kv8_attn: verification attention over the paged 8-bit cache, and the
// weight that each cached token received.
#include <algorithm>
#include <cmath>

#include "kv8.cuh"
#include "kv8_attn.cuh"

FC_DEFINE_ERROR_WORD(kv8_attn)

namespace {

constexpr int HD = KV8_D;

// ---------------------------------------------------------------------------
// Few query rows for a kv head (n_pad * H / Hkv <= 16: single tokens, small
// trees).  The cache's read bounds this; next to it, what it costs to turn 8-bit
// numbers into tensor-core operands.  32 tokens over 16384 keys, 8 kv heads, take
// 168 us (6.4 TB/s), one over 131071 51 (5.3; 5 of them start and join), one
// over 500 7.9 (latency); 24 x 4 nodes over up to 8192 keys 54, two tiles of rows with 8 warps an
// SM for want of registers.
//
// Keys and dimensions are the rows of mma.m16n8k16 (operand A, from the
// cache), query rows its 8 columns:
//   S^T [16 keys][8 rows] = K Q^T,   O^T [128 dims][8 rows] += V^T P^T
// in fp16, which holds every e4m3 number.
//   * Queries enter as fp16 times one power of two for the unit (its largest
//     query value below 2^15); the block's scale multiplies a key's scores.
//   * The second product takes w = 2^(z - m) * (value scale) in fp16.  The
//     row's reference m (O and the row sum are relative to it) moves when a w
//     passes 2^15, to where the largest is 2^11 to 2^12: a running maximum of
//     z + log2(value scale), moved lazily.  (High in fp16's range, so that a
//     weight of 2^-25 of the largest keeps 11 bits.)  For the
//     reference a value scale counts as at least 2^-80, so that 2^(z - m), and
//     the row sum, stay in fp32's range where a row of V is all zeros.  The
//     test for the move is that w is NOT below 2^15: far above the reference
//     2^(z - m) is infinite and its product with a scale of 0 NaN.
// A warp takes every FEW_WARPS-th step of 32 keys (8 KB, two blocks of 16 rows
// in a page), three steps in flight by 16-byte asynchronous copies.  S^T
// becomes P^T's operand by 8x8 transposes in registers.
//
// Dimensions 32t .. 32t + 31 (t = lane % 4) are the lane's part of K, 16g ..
// 16g + 15 (g = lane / 4) its part of V, each as they lie in memory; the queries
// are permuted to match.
// ---------------------------------------------------------------------------
constexpr int FEW_WARPS = 4, FEW_THREADS = FEW_WARPS * 32, FEW_CTAS = 2;
constexpr int STEP = 32;         // keys a step
constexpr int FEW_STAGES = 3;    // steps in flight a warp
constexpr int OFF_VROWS = STEP * HD, OFF_SC = 2 * STEP * HD;
constexpr int STEP_BYTES = OFF_SC + 128;
// A unit's start and end in steps of a CTA; parts of at least 8 steps (1 x 2000
// keys take 9.1 us, in parts of 16 10.9, of 4 8.5, but 1 x 131071 and the ragged
// shapes no less); a unit of fewer than CUT_STEPS stays whole (1 x 500 keys 7.7 us, in
// two parts 8.7).  A unit's cost: with 8 instead of 16, 24 ragged requests of up
// to 8192 keys 59 us instead of 54.
constexpr int UNIT_COST = 16, PART_STEPS = 8, CUT_STEPS = 24;
constexpr float W_MAX = 32768.f;
constexpr int VS_MIN_EXP = -80;
constexpr float VS_MIN = 0x1p-80f;
// A reference before any key: 2^(z + 1e30) is infinite and not below W_MAX
// whatever it is multiplied by, 2^(-1e30 - m) is 0.
constexpr float M_START = -1e30f;
constexpr float F32_MAX = 0x1.fffffep127f;
template <int NT>
struct FewSmem {
  static constexpr int ROWS = 8 * NT;
  static constexpr int RING = FEW_WARPS * FEW_STAGES * STEP_BYTES;
  static constexpr int OUT_PITCH = HD + 4;  // floats a row of a warp's partial
  static constexpr int MERGE = FEW_WARPS * ROWS * (OUT_PITCH + 2) * 4;
  static constexpr int JOIN = (ROWS * 152 * FEW_CTAS + FEW_THREADS * 4) * 4;  // pieces' weights, subsets' sums
  // the new tokens' keys, values and masks (a row of 256 bytes at 272, so that
  // eight rows' reads fall in different banks)
  static constexpr int NEW_PITCH = HD * 2 + 16, NEW = 2 * 16 * NEW_PITCH + 16 * 8;
  static constexpr int OFF_NEW = RING > MERGE ? (RING > JOIN ? RING : JOIN) : (MERGE > JOIN ? MERGE : JOIN);
  static constexpr int BYTES = OFF_NEW + NEW;
};

struct FewArgs {
  Kv8Args a;
  int split;         // 1: units are cut anywhere, by steps; 0: a CTA takes whole units
  uint32_t by_G;     // r / G is r * by_G >> 16 for r < 16
  int* cnt;          // [grid] arrivals at the cut unit that begins in a CTA (at most one does), zero between calls
  float* part;       // [grid][2][ROWS][HD + 2]: O unnormalised, m, l of a CTA's first and last piece
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n" ::"r"(dst), "l"(src) : "memory");
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
// Two e4m3 numbers (the low 16 bits) as fp16; exact.
__device__ __forceinline__ uint32_t e4m3x2_f16x2(uint32_t two) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(two));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x2_f16x2_hi(uint32_t two) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(r) : "r"(two));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float min_nan(float a, float b) {  // NaN of either
  float d;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
// l * 2^d by two factors: a row's sum, relative to a reference that value scales move, may be 2^112 and d -180
__device__ __forceinline__ float times_pow2(float l, float d) {
  const float h = exp2_fast(0.5f * d);
  return l * h * h;
}
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ int expo(float x) { return (int)((__float_as_uint(x) >> 23) & 255u) - 127; }
__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// A staged step keeps row r's 16-byte chunk c at r * 128 + (c ^ (r % 8)) * 16,
// such that a quarter warp's 16-byte reads of the keys (rows g and g + 1, every
// second chunk) and of the values (rows 2t, t = 0..3, two chunks) each fall in
// different banks.

// steps of a length up to 2^31 - 1, whose rounding up passes an int
__device__ __forceinline__ int steps_of(int kvl) { return (int)(((uint32_t)kvl + STEP - 1) / STEP); }

__device__ __forceinline__ int few_steps(const Kv8Args& a, int b, int& nn, int& kvl, bool& bad) {
  kvl = a.kv_len[b];
  nn = a.n_nodes ? a.n_nodes[b] : a.n_pad;
  bad = nn < 0 || nn > a.n_pad || kvl < 0 || kvl > (long long)a.max_pages << a.shift;
  if (bad) nn = kvl = 0;
  return nn == 0 ? 1 : max(1, steps_of(kvl) + (a.k_new ? 1 : 0));
}

// parts that a unit of so many steps is worth (0: like 1)
__device__ __forceinline__ int parts_of(int steps) { return steps < CUT_STEPS ? 0 : steps / PART_STEPS; }

template <int NT>
__global__ void __launch_bounds__(FEW_THREADS, FEW_CTAS) k_kv8_attn_few(FewArgs f) {
  using L = FewSmem<NT>;
  extern __shared__ __align__(1024) unsigned char smem[];
  __shared__ int s_last;
  const Kv8Args& a = f.a;
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
  KvCut cut(1, 1, 1);
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
    cut = KvCut(__reduce_add_sync(0xFFFFFFFFu, sum) * a.Hkv, gridDim.x, UNIT_COST + PART_STEPS);
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
    const float* sc_lane = (lane & 2) ? a.vs : a.ks;
    const uint32_t put0 = ring + (lane >> 3) * 128 + (((lane & 7) ^ (lane >> 3)) << 4);
    // ---- cached steps of this warp: s0 + warp, s0 + warp + 8, ...
    const int cs1 = min(s1, c_steps);
    const int n_it = cs1 > s0 + warp ? (cs1 - s0 - warp + FEW_WARPS - 1) / FEW_WARPS : 0;
    int id_a = 0, id_b = 0;  // page ids of the two runs of 16 keys of the warp's next 32 steps, one a lane
    uint32_t outside = 0;    // bits 2 x stage, + 1: that run's page is not in the pool
    const int32_t* tab = a.table + (size_t)b * a.max_pages;
    // runs of 16 rows, a scale each, are counted in 32 bits
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
        const uint32_t d0 = put0 + at, d1 = d0 ^ 64u;
        const uint8_t *ka = k_lane + (uint64_t)ra * 2048u, *kb = k_lane + (uint64_t)rb * 2048u;
        const uint8_t *va = v_lane + (uint64_t)ra * 2048u, *vb = v_lane + (uint64_t)rb * 2048u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // four rows each
          const uint32_t d = ((j & 1) ? d1 : d0) + j * 512;
          cp_async16(d, ka + j * 512);
          cp_async16(d + 2048, kb + j * 512);
          cp_async16(d + OFF_VROWS, va + j * 512);
          cp_async16(d + OFF_VROWS + 2048, vb + j * 512);
        }
        if (lane < 4)  // K scales of the two runs, then V scales
          cp_async4(ring + at + OFF_SC + lane * 4, sc_lane + ((lane & 1) ? rb : ra));
      }
      cp_async_commit();
    };
    // ---- queries: the unit's power of two, then the operand registers
    // k-step j: dimensions 32t + 4j .. + 3 of a key's 32-byte quarter t
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
    const int qe = top ? max((int)(top >> 7) - 127, -100) : 0;  // largest |q| < 2^(qe + 1)
    const float q_mul = pow2i(14 - qe);
    const float z_mul = a.scale_log2 * pow2i(qe - 14);
    uint32_t qf[NT][8][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 w = qw[n][i];
        qf[n][2 * i][0] = pack_f16x2(lo_f(w.x) * q_mul, hi_f(w.x) * q_mul);
        qf[n][2 * i][1] = pack_f16x2(lo_f(w.y) * q_mul, hi_f(w.y) * q_mul);
        qf[n][2 * i + 1][0] = pack_f16x2(lo_f(w.z) * q_mul, hi_f(w.z) * q_mul);
        qf[n][2 * i + 1][1] = pack_f16x2(lo_f(w.w) * q_mul, hi_f(w.w) * q_mul);
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
          for (int i = 0; i < 4; ++i) {
            const int e = expo(vs[i]);  // 128: NaN, whose row is NaN whatever the reference; its powers still count
            top = fmaxf(top, fmaf(d[i][r], ks[i], (float)((e == 128 ? VS_MIN_EXP : max(e, VS_MIN_EXP)) - 11)));
          }
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
          const float mn = fmaxf(m[n][r], top), al = exp2_fast(m[n][r] - mn);
          l[n][r] = times_pow2(l[n][r], m[n][r] - mn);
          m[n][r] = mn;
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
      const float4 sc = *reinterpret_cast<const float4*>(st + OFF_SC);
      // (finite: a sum of 0 between large queries and large keys is a score of 0)
      const float ka = min_nan(sc.x * z_mul, F32_MAX), kb = min_nan(sc.y * z_mul, F32_MAX);
      float ks[4] = {ka, ka, kb, kb};
      float vs[4] = {sc.z, sc.z, sc.w, sc.w};
      float z[NT][4][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {  // keys 16h + g, 16h + 8 + g
        float d[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) d[n][0] = d[n][1] = d[n][2] = d[n][3] = 0.f;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const unsigned char* at = st + h * 2048 + g * 128 + (((2 * t + c) ^ g) << 4);
          const uint4 k0 = *reinterpret_cast<const uint4*>(at), k1 = *reinterpret_cast<const uint4*>(at + 1024);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = (&k0.x)[i], y = (&k1.x)[i];
            const uint32_t x0 = e4m3x2_f16x2(x), x1 = e4m3x2_f16x2_hi(x), y0 = e4m3x2_f16x2(y), y1 = e4m3x2_f16x2_hi(y);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_f16(d[n], x0, y0, x1, y1, qf[n][4 * c + i][0], qf[n][4 * c + i][1]);
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
          const int j = 8 * i + g;
          if (j >= left || ((out_now >> (j >> 4)) & 1u)) {
            vs[i] = 0.f;
            ks[i] = 1.f;
#pragma unroll
            for (int n = 0; n < NT; ++n) z[n][i][0] = z[n][i][1] = -INFINITY;
          }
        }
        // nor may their values be NaN, which no weight of 0 takes out
#pragma unroll 1
        for (int j = 0; j < STEP; ++j)
          if (j >= left || ((out_now >> (j >> 4)) & 1u))
            reinterpret_cast<uint32_t*>(smem + (ring_p - smem) + stage * STEP_BYTES + OFF_VROWS)[j * 32 + lane] = 0u;
        __syncwarp();
      }
      if (a.z) {  // the scores, for the weights
        const long long key = kvl - left + g;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            if (8 * n + 2 * t + r >= R) continue;
            float* to = a.z + (((size_t)b * a.Hkv + gh) * a.R + 8 * n + 2 * t + r) * a.z_stride + key;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (8 * i + g < left) to[8 * i] = z[n][i][r] * ks[i];
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
      // O^T: k 2t, 2t + 1, 2t + 8, 2t + 9 of product h are those of its 16 keys
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const unsigned char* at = st + OFF_VROWS + h * 2048 + t * 256;
        const uint4 va = *reinterpret_cast<const uint4*>(at + ((g ^ (2 * t)) << 4));
        const uint4 vb = *reinterpret_cast<const uint4*>(at + 128 + ((g ^ (2 * t + 1)) << 4));
        const uint4 vc = *reinterpret_cast<const uint4*>(at + 1024 + ((g ^ (2 * t)) << 4));
        const uint4 vd = *reinterpret_cast<const uint4*>(at + 1024 + 128 + ((g ^ (2 * t + 1)) << 4));
#pragma unroll
        for (int u = 0; u < 4; ++u) {  // four dims: a word of each key's chunk
          const uint32_t x = (&va.x)[u], y = (&vb.x)[u], z0 = (&vc.x)[u], w0 = (&vd.x)[u];
          // (dim of key 2t, dim of key 2t + 1) in 16 bits, two dims a word
          const uint32_t xa = __byte_perm(x, y, 0x5140), xb = __byte_perm(x, y, 0x7362);
          const uint32_t za = __byte_perm(z0, w0, 0x5140), zb = __byte_perm(z0, w0, 0x7362);
          const uint32_t a0 = e4m3x2_f16x2(xa), a1 = e4m3x2_f16x2_hi(xa), a2 = e4m3x2_f16x2(za), a3 = e4m3x2_f16x2_hi(za);
          const uint32_t c0 = e4m3x2_f16x2(xb), c1 = e4m3x2_f16x2_hi(xb), c2 = e4m3x2_f16x2(zb), c3 = e4m3x2_f16x2_hi(zb);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma_f16(o[n][2 * u], a0, a1, a2, a3, pb[n][2 * h], pb[n][2 * h + 1]);
            mma_f16(o[n][2 * u + 1], c0, c1, c2, c3, pb[n][2 * h], pb[n][2 * h + 1]);
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
        pb[n][0] = transpose8x8(pack_bf16x2(w[0][0], w[0][1]));
        pb[n][1] = transpose8x8(pack_bf16x2(w[1][0], w[1][1]));
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
          const uint32_t a0 = __byte_perm((&v[0].x)[u], (&v[1].x)[u], 0x5410), a1 = __byte_perm((&v[0].x)[u], (&v[1].x)[u], 0x7632);
          const uint32_t a2 = __byte_perm((&v[2].x)[u], (&v[3].x)[u], 0x5410), a3 = __byte_perm((&v[2].x)[u], (&v[3].x)[u], 0x7632);
#pragma unroll
          for (int n = 0; n < NT; ++n) mma_bf16(o[n][4 * h + u], a0, a1, a2, a3, pb[n][0], pb[n][1]);
        }
      }
      bad = __reduce_or_sync(0xFFFFFFFFu, bad);
      if (bad) {  // NaN in the rows' sums of values, not in their sums of powers, which the weights go by
        uint32_t rows_bad = 0;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (((seen >> (4 * n + c)) & 1u) && ((bad >> (g + 8 * (c >> 1))) & 1u)) rows_bad |= 1u << (8 * n + 2 * t + (c & 1));
        rows_bad = __reduce_or_sync(0xFFFFFFFFu, rows_bad);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int r = 0; r < 2; ++r)
            if ((rows_bad >> (8 * n + 2 * t + r)) & 1u)
#pragma unroll
              for (int mt = 0; mt < 8; ++mt) o[n][mt][r] = o[n][mt][2 + r] = __uint_as_float(0x7FC00000u);
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
        float* dst = po + row * L::OUT_PITCH + 16 * g;
#pragma unroll
        for (int mt = 0; mt < 8; mt += 2)
          *reinterpret_cast<float4*>(dst + 2 * mt) = make_float4(o[n][mt][r], o[n][mt][2 + r], o[n][mt + 1][r], o[n][mt + 1][2 + r]);
        if (g == 0) pml[row] = make_float2(m[n][r], sum);
      }
    __syncthreads();
    const bool whole = s0 == 0 && s1 == steps;
    const int rows_all = a.n_pad * a.G;  // rows past the nodes are written as zeros
    float* slot = piece(blockIdx.x);
    auto lse_of = [&](int r, float m, float sum) {
      a.lse[((size_t)b * a.Hkv + gh) * a.R + r] = sum == 0.f ? INFINITY : m + log2f(sum);
    };
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
        sum += times_pow2(ml.y, ml.x - mx);
        acc.x += v.x * k, acc.y += v.y * k, acc.z += v.z * k, acc.w += v.w * k;
      }
      if (whole) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (a.z && d4 == 0) lse_of(r, mx, sum);
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
            sum = times_pow2(sum, mx - mn) + times_pow2(ml.y, ml.x - mn);
            mx = mn;
            wt[r * nc + c] = ml.x;
          }
          float all = mx;
#pragma unroll
          for (int x = 16; x > 0; x >>= 1) all = fmaxf(all, __shfl_xor_sync(0xFFFFFFFFu, all, x));
          sum = times_pow2(sum, mx - all);
#pragma unroll
          for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          if (a.z && lane == 0) lse_of(r, all, sum);
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

constexpr int FEW_GRID = 152 * FEW_CTAS;

static_assert(FEW_GRID * sizeof(int) <= KV8_WS_COUNTERS, "room for the counters");

template <int NT>
fc_status launch_few(const Kv8Args& a, void* ws, size_t ws_bytes, cudaStream_t s) {
  static std::atomic<unsigned long long> done{0};
  const fc_status st = fc_once_per_device(done, [](int) {
    return fc_cuda_status(cudaFuncSetAttribute(k_kv8_attn_few<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               FewSmem<NT>::BYTES));
  });
  if (st != FC_OK) return st;
  const int full = FEW_GRID;
  const size_t cnt = KV8_WS_COUNTERS, one = (size_t)2 * FewSmem<NT>::ROWS * (HD + 2) * sizeof(float);
  const long long units = (long long)a.B * a.Hkv;
  // at most what the tables could hold, in steps (past 32 bits there are units enough without cutting them)
  const long long longest = (((long long)a.max_pages << a.shift) + STEP - 1) / STEP + 1, most = units * (longest + UNIT_COST);
  int grid = (int)std::min<long long>(full, units * std::max<long long>(1, longest / PART_STEPS));
  FewArgs f{a, 1, 65536u / a.G + 1, nullptr, nullptr};
  if (ws && ws_bytes > cnt) grid = (int)std::min<size_t>(grid, (ws_bytes - cnt) / one);
  // a workspace for fewer CTAs than whole units would fill: whole units (16 x 8000 keys, 8 kv heads, on
  // two CTAs 2.81 ms, whole units 0.05)
  if (!ws || ws_bytes <= cnt || grid < std::min<long long>(full, units) || most > 0x7FFFFFFFll) {
    f.split = 0;
    grid = (int)std::min<long long>(units, 1 << 20);
  } else {
    f.cnt = static_cast<int*>(ws);
    f.part = reinterpret_cast<float*>(static_cast<unsigned char*>(ws) + cnt);
  }
  k_kv8_attn_few<NT><<<grid, FEW_THREADS, FewSmem<NT>::BYTES, s>>>(f);
  return FC_CHECK_LAUNCH();
}

// weight = decay * weight + the sum over a kv head's rows of 2^(score - log2 of
// the row's sum): the scores that the attention left, four keys a thread.  (A
// row's sum is known only when all its keys are done.  24 x 16 rows of up to 8192
// keys: 14 us, most of it the scores' read.)
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

// at most 2^30 query rows over all heads (the product of all three may pass 64 bits)
bool rows_ok(int batch, int n_pad, int H) { return batch <= (1ll << 30) / ((long long)H * n_pad); }

// bytes of the scores and of the rows' sums that the weights are made from
size_t score_bytes(long long batch, int n_pad, int H, long long keys) {
  const size_t rows = (size_t)batch * n_pad * H;
  return (rows * (size_t)keys * 4 + rows * 4 + 255) & ~(size_t)255;
}

}  // namespace

extern "C" size_t fc_kv8_attn_workspace(int batch, int n_pad, int H, int Hkv, int64_t weight_keys) {
  if (batch < 1 || !shape_ok(n_pad, H, Hkv) || !rows_ok(batch, n_pad, H) || weight_keys < 0 || weight_keys > 0x7FFFFFFFll ||
      (weight_keys && n_pad * (H / Hkv) > 16))
    return 0;
  if (n_pad * (H / Hkv) > 16) return kv8_attn_many_workspace(batch, n_pad, H, Hkv);
  return KV8_WS_COUNTERS + (size_t)FEW_GRID * 2 * FewSmem<2>::ROWS * (HD + 2) * sizeof(float) +
         (weight_keys ? score_bytes(batch, n_pad, H, weight_keys) : 0);
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
  if (!rows_ok(batch, n_pad, H) || (long long)max_pages << shift > 0x7FFFFFFFll || (d_weight && n_pad * G > 16))
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
    if (!d_ws || ws_bytes < fc_kv8_attn_workspace(batch, n_pad, H, cache->Hkv, a.z_stride)) return FC_ERR_WORKSPACE;
    if (batch * cache->Hkv > 65535) return FC_ERR_UNSUPPORTED;
    ws_bytes = ws_bytes / 256 * 256 - need;  // the scores lie at its end
    a.z = reinterpret_cast<float*>(static_cast<unsigned char*>(d_ws) + ws_bytes);
    a.lse = a.z + (size_t)batch * n_pad * H * a.z_stride;
  }
  fc_status st = FC_OK;
  if (a.R <= 8) st = launch_few<1>(a, d_ws, ws_bytes, s);
  else if (a.R <= 16) st = launch_few<2>(a, d_ws, ws_bytes, s);
  else st = kv8_attn_many(a, d_ws, ws_bytes, s);
  if (st != FC_OK) return st;
  if (d_weight) {
    const dim3 grid((unsigned)std::min<long long>((a.z_stride + 1023) / 1024, 1024), (unsigned)(batch * cache->Hkv));
    k_kv8_weights<<<grid, 256, 0, s>>>(a, d_weight, decay);
  }
  return FC_CHECK_LAUNCH();
}
