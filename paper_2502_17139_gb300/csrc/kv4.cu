// The paged 4-bit KV cache: block tables and slot maps built from request
// lengths (fc_kv_pages_plan, fc_kv_pages_release), and keys and values
// quantised into the pages and read back (fc_kv4_write, fc_kv4_read).
//
// A cached row x (128 values of one token and kv head) is held as
//   s = bf16(max|x| / 7),  c_d = clamp(rint(x_d / s), -7, 7)  (ties to even; all 0 when s = 0),
// the numbers c_d + 8 two to a byte (dimension 2i in byte i's low half), and
// stands for c_d * s.  One scale a row keeps both attention products exact in
// the tensor cores: a number in -7..7 is a bf16 value, and the scale
// multiplies a whole key's score or probability instead of its 128 elements.
#include <algorithm>

#include "fc_common.cuh"
#include "kv4.cuh"

FC_DEFINE_ERROR_WORD(kv4)

namespace {

constexpr int HD = KV4_D;

// ---------------------------------------------------------------------------
// Pages.
// ---------------------------------------------------------------------------
constexpr int PL_MAX_THREADS = 1024;  // a CTA has a thread for each request of a chunk
constexpr int PL_ROWS = 2;            // rows a thread takes at least, once there are CTAs for every SM

struct PlanArgs {
  const int32_t *kv_len, *n_new;
  int batch, shift, max_pages;
  int32_t* table;
  const int32_t* free_list;
  int n_pages;
  const int32_t* n_free_in;
  const int32_t* path;
  int path_cap, n_per_seq, rows_cap;
  int32_t *cu, *seq, *pos, *slot, *src, *kv_out, *n_free_out;
  unsigned int* err;
};

// Inclusive sums of two values over the block's threads (64-bit: lengths are
// the caller's data, and their sum may pass 32 bits before it is refused).
__device__ __forceinline__ void block_scan2(long long& a, long long& b, long long (*s_part)[2]) {
  const int lane = threadIdx.x & 31, wp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xFFFFFFFFu, a, o), y = __shfl_up_sync(0xFFFFFFFFu, b, o);
    if (lane >= o) a += x, b += y;
  }
  if (warps == 1) return;
  if (lane == 31) s_part[wp][0] = a, s_part[wp][1] = b;
  __syncthreads();
  // every warp sums the warps' totals for itself
  long long ta = lane < wp ? s_part[lane][0] : 0, tb = lane < wp ? s_part[lane][1] : 0;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    ta += __shfl_xor_sync(0xFFFFFFFFu, ta, o);
    tb += __shfl_xor_sync(0xFFFFFFFFu, tb, o);
  }
  a += ta, b += tb;
}

// Every CTA sums over all requests itself, a chunk (a thread each) at a time,
// and fills its own rows and its own requests' table entries, so one launch
// does the whole plan with no CTA waiting for another.  The lengths are a few
// KB that L2 serves; bound by latency at every size that a step has: 6 us for
// 32 requests, 8 us for 1000 with 243,000 new tokens.
__global__ void __launch_bounds__(PL_MAX_THREADS) k_pages_plan(PlanArgs a, int rows_per_cta) {
  __shared__ long long s_part[PL_MAX_THREADS / 32][2];
  __shared__ long long s_sum[2];
  __shared__ int32_t s_cu[PL_MAX_THREADS + 1], s_off[PL_MAX_THREADS], s_more[PL_MAX_THREADS];
  __shared__ int2 s_kv[PL_MAX_THREADS];  // length, pages held
  const int tid = threadIdx.x, chunk = blockDim.x;
  const long long page = 1ll << a.shift;
  const int in_page = (1 << a.shift) - 1;
  int n_free = *a.n_free_in;
  const int r_lo = (int)min((long long)blockIdx.x * rows_per_cta, (long long)a.rows_cap);
  const int r_hi = (int)min((long long)r_lo + rows_per_cta, (long long)a.rows_cap);
  if (n_free < 0 || n_free > a.n_pages) {
    if (blockIdx.x == 0 && tid == 0) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_INVALID);
    n_free = 0;
  }
  long long row_base = 0, page_base = 0;
  long long taken = 0;  // pages of the requests served so far (CTA 0)
  for (int b0 = 0; b0 < a.batch; b0 += chunk) {
    const int b = b0 + tid;
    long long kv = 0, n = 0;
    const bool ok = b < a.batch;
    bool bad = false;
    if (ok) {
      kv = a.kv_len[b];
      n = a.n_new[b];
      bad = kv < 0 || n < 0;
      kv = max(kv, 0ll);
      n = max(n, 0ll);
    }
    const long long have = (kv + page - 1) >> a.shift, need = (kv + n + page - 1) >> a.shift;
    const bool fits = ok && !bad && need <= a.max_pages && kv + n <= 0x7FFFFFFFll;
    long long rows_end = n, page_end = fits ? need - have : 0;
    const long long more = page_end;
    block_scan2(rows_end, page_end, s_part);
    rows_end += row_base;
    page_end += page_base;
    const bool served = fits && rows_end <= a.rows_cap && (more == 0 || page_end <= n_free);
    if (ok) {
      s_cu[tid + 1] = (int32_t)min(rows_end, (long long)a.rows_cap);
      s_kv[tid] = make_int2((int32_t)kv, (int32_t)have);
      s_off[tid] = (int32_t)min(page_end - more, (long long)n_free);
      s_more[tid] = served ? (int32_t)more : -1;
    }
    if (tid == 0) s_cu[0] = (int32_t)min(row_base, (long long)a.rows_cap);
    if (tid == chunk - 1) s_sum[0] = rows_end, s_sum[1] = page_end;
    if (blockIdx.x == 0 && ok) {
      a.cu[b + 1] = (int32_t)min(rows_end, (long long)a.rows_cap);
      a.kv_out[b] = (int32_t)(served ? kv + n : kv);
      if (b == 0) a.cu[0] = 0;
      if (!served) fc_flag(FC_ERR_WORD(a.err), bad ? FC_EBIT_INVALID : FC_EBIT_CAPACITY);
      taken += served ? more : 0;
    }
    const int in_chunk = min(chunk, a.batch - b0);
    __syncthreads();
    row_base = s_sum[0];
    page_base = s_sum[1];
    // rows of this chunk's requests in [r_lo, r_hi)
    const int lo = max(r_lo, s_cu[0]), hi = min(r_hi, s_cu[in_chunk]);
#pragma unroll 2
    for (int r = lo + tid; r < hi; r += chunk) {
      int x = 0;  // s_cu[x] <= r < s_cu[x + 1]
#pragma unroll 1
      for (int step = 512; step > 0; step >>= 1)
        if (x + step < in_chunk && s_cu[x + step] <= r) x += step;
      const int q = b0 + x, j = r - s_cu[x];
      const int2 kh = s_kv[x];
      const int p = (int)((uint32_t)kh.x + (uint32_t)j);
      int sl = -1;
      if (s_more[x] >= 0) {
        const int pg = p >> a.shift;
        const int id = pg < kh.y ? a.table[(size_t)q * a.max_pages + pg] : a.free_list[n_free - 1 - s_off[x] - (pg - kh.y)];
        const bool in = (unsigned)id < (unsigned)a.n_pages;
        sl = in ? (id << a.shift) + (p & in_page) : -1;
        if (!in) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_INVALID);
      }
      a.seq[r] = q;
      a.pos[r] = p;
      a.slot[r] = sl;
      if (a.src) {
        const int node = a.path ? (j < a.path_cap ? a.path[(size_t)q * a.path_cap + j] : -1) : j;
        a.src[r] = node < 0 || node >= a.n_per_seq ? -1 : q * a.n_per_seq + node;
      }
    }
    // table entries of new pages: 8 lanes a request
    for (int i = (tid >> 3) * gridDim.x + blockIdx.x; i < in_chunk; i += (chunk >> 3) * gridDim.x) {
      const int m = s_more[i];
      for (int j = tid & 7; j < m; j += 8)
        a.table[(size_t)(b0 + i) * a.max_pages + s_kv[i].y + j] = a.free_list[n_free - 1 - s_off[i] - j];
    }
    __syncthreads();  // the chunk's arrays are read
  }
  // rows past the last request's
  const int total = (int)min(row_base, (long long)a.rows_cap);
  for (int r = max(r_lo, total) + tid; r < r_hi; r += chunk) {
    a.seq[r] = -1;
    a.pos[r] = -1;
    a.slot[r] = -1;
    if (a.src) a.src[r] = -1;
  }
  if (blockIdx.x == 0) {
    long long t2 = 0;
    block_scan2(taken, t2, s_part);
    if (tid == chunk - 1) *a.n_free_out = n_free - (int32_t)taken;
    if (a.batch == 0 && tid == 0) a.cu[0] = 0;
  }
}

constexpr int PL_THREADS = 512;  // of the release

// One CTA: the pages of request b past ceil(keep / page) go back on the free
// list in request order.  4 to 5 us for 32 requests, 8 us for one of 1000 that
// gives back 256 pages (latency), 91 us for 256,000 pages at once.
__global__ void __launch_bounds__(PL_THREADS) k_pages_release(const int32_t* kv_len, const int32_t* keep, int batch,
                                                              int shift, const int32_t* table, int max_pages,
                                                              int32_t* free_list, int n_pages,
                                                              const int32_t* n_free_in, int32_t* n_free_out,
                                                              int32_t* kv_out, unsigned int* err) {
  __shared__ long long s_part[PL_THREADS / 32][2];
  __shared__ long long s_base;
  __shared__ int32_t s_first[PL_THREADS], s_n[PL_THREADS], s_at[PL_THREADS];
  const int tid = threadIdx.x;
  const long long page = 1ll << shift;
  int n_free = *n_free_in;
  bool flag = n_free < 0 || n_free > n_pages;
  if (flag) n_free = n_pages;  // nothing can be given back
  if (tid == 0) s_base = n_free;
  __syncthreads();
  for (int b0 = 0; b0 < batch; b0 += PL_THREADS) {
    const int b = b0 + tid;
    long long first = 0, n = 0, kv = 0, kp = 0;
    if (b < batch) {
      kv = kv_len[b];
      kp = keep[b];
      if (kv < 0 || kp < 0) flag = true;
      kv = std::max(kv, 0ll);
      kp = std::min(std::max(kp, 0ll), kv);
      first = (kp + page - 1) >> shift;
      const long long held = (kv + page - 1) >> shift;
      if (held > max_pages) flag = true;
      n = std::max(std::min<long long>(held, max_pages) - first, 0ll);
    }
    long long end = n, dummy = 0;
    block_scan2(end, dummy, s_part);
    const long long base = s_base;
    const bool fits = b < batch && base + end <= n_pages;  // else the tables are not this pool's
    if (b < batch) {
      if (!fits && n > 0) flag = true;
      kv_out[b] = (int32_t)(fits ? kp : kv);
    }
    s_first[tid] = (int32_t)first;
    s_n[tid] = fits ? (int32_t)n : 0;
    s_at[tid] = fits ? (int32_t)(base + end - n) : 0;
    __syncthreads();
    for (int i = tid >> 5; i < min(PL_THREADS, batch - b0); i += PL_THREADS / 32)  // a warp a request
      for (int j = tid & 31; j < s_n[i]; j += 32)
        free_list[s_at[i] + j] = table[(size_t)(b0 + i) * max_pages + s_first[i] + j];
    // the requests that fit are a prefix of those with pages to give
    long long given = fits ? n : 0, d2 = 0;
    block_scan2(given, d2, s_part);
    __syncthreads();
    if (tid == PL_THREADS - 1) s_base = base + given;
    __syncthreads();
  }
  if (flag) fc_flag(FC_ERR_WORD(err), FC_EBIT_INVALID);
  if (tid == 0) *n_free_out = (*n_free_in < 0 || *n_free_in > n_pages) ? 0 : (int32_t)s_base;
}

// ---------------------------------------------------------------------------
// Write and read.
// ---------------------------------------------------------------------------
constexpr int WR_THREADS = 128, WR_CTAS = 16;  // all of an SM's 2048 threads: what is in flight hides HBM's latency
constexpr int WR_LANES = HD / 8;                     // lanes a row: 8 dimensions (16 bytes of bf16) each
constexpr int WR_GROUPS = WR_THREADS / WR_LANES;     // rows in flight a CTA

constexpr long long MAX_ITEMS = 1ll << 30;           // rows times heads a call (their counters are 32-bit)

struct KvRows {
  const __nv_bfloat16 *k, *v;
  int n_per_seq, n_src;
  bool one_seq;  // the rows are one sequence: no division
  long long seq_stride, row_stride, head_stride;
};

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// 8 values of a row (4 words of two) to 8 numbers of 4 bits, given the row's
// scale.  x * (1 / s) is rounded onto a grid of 2^-11 before the rounding to
// whole numbers.  x and s have 8 significant bits: with x = X 2^a, s = S 2^b
// (X, S in 128..255) the quotient's distance from a tie (2k+1)/2 is
// |2X 2^(a-b) - (2k+1) S| / 2S, and near a tie of at most 7.1 a - b >= -2, so
// the numerator is 0 or at least 1/2 and the distance 0 or above 2^-10.  The
// grid holds every tie and moves a value by at most 2^-12, the reciprocal is
// good to 2^-22, so this is rint(x / s) exactly, in two operations (the second
// adds what rounds to whole numbers, less the grid's constant) where a division
// takes about ten.  A byte's two numbers are put together as
// 16 hi + lo in fp32 too (the integer pipe has half the rate), and taken from
// the sum's lowest eight bits.
__device__ __forceinline__ uint32_t quantise8(const uint4& x, float s) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  if (s >= 0x1p-100f && s <= 0x1p100f) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    constexpr float GRID = 6144.f;       // 1.5 * 2^12: neighbours are 2^-11 apart
    constexpr float WHOLE = 12582912.f;  // 1.5 * 2^23: neighbours are 1 apart, the low byte is 0
    uint32_t byte[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float lo = __fadd_rn(__fmaf_rn(lo_f(w[i]), r, GRID), WHOLE + 8.f - GRID);
      const float hi = __fadd_rn(__fmaf_rn(hi_f(w[i]), r, GRID), WHOLE + 8.f - GRID);
      byte[i] = __float_as_uint(__fmaf_rn(__fadd_rn(hi, -WHOLE), 16.f, lo));
    }
    return __byte_perm(__byte_perm(byte[0], byte[1], 0x0040), __byte_perm(byte[2], byte[3], 0x0040), 0x5410);
  }
  uint32_t out = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = s > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(lo_f(w[i]), s)), -7.f), 7.f) : 0.f;
    const float b = s > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(hi_f(w[i]), s)), -7.f), 7.f) : 0.f;
    out |= (uint32_t)((int)a + 8) << (8 * i);
    out |= (uint32_t)((int)b + 8) << (8 * i + 4);
  }
  return out;
}

// A lane group's (row, head) items, the grid's stride apart, without a division
// an item.  A CTA's eight follow one another, so that the 16-bit side is read
// (and written) in pieces of 2 KB; the other way round, eight rows of one head,
// which makes the 4-bit side contiguous, reads back 65000 x 8 rows in 75 us
// instead of 63.
struct Items {
  int r, h, dr, dh;
  __device__ __forceinline__ Items(int Hkv) {
    const int first = blockIdx.x * WR_GROUPS + threadIdx.x / WR_LANES, stride = gridDim.x * WR_GROUPS;
    r = first / Hkv;
    h = first - r * Hkv;
    dr = stride / Hkv;
    dh = stride - dr * Hkv;
  }
  __device__ __forceinline__ void next(int Hkv) {
    r += dr;
    h += dh;
    if (h >= Hkv) h -= Hkv, ++r;
  }
};

// 16 lanes a (row, head), key and value: the largest magnitude from the bf16
// bits (as unsigned numbers they order like the magnitudes, infinities and NaN
// on top), the scale, the numbers.  65000 x 8 rows written and read back take
// 124 us, 4.8 TB/s of the 0.6 GB in and out, 66 of them the write (a copy's rate
// gives 47), which issues in 80% of the cycles; two or four items a lane group at
// a time, with fewer threads for it, took 134 to 153 us.
// bf16(top / 7) is taken as bf16(top * fl(1/7)): top has 8 significant bits,
// so top / 7 is no midpoint of two bf16 values and lies 2^-15 of itself or
// more from one, the product's error is 2^-23 of it.
__global__ void __launch_bounds__(WR_THREADS, WR_CTAS) k_kv4_write(KvRows x, const int32_t* __restrict__ src,
                                                          const int32_t* __restrict__ slot, int rows, int Hkv,
                                                          int shift, long long n_slots, uint32_t* __restrict__ kc,
                                                          uint32_t* __restrict__ vc, __nv_bfloat16* __restrict__ ks,
                                                          __nv_bfloat16* __restrict__ vs, unsigned int* err) {
  const int lane = threadIdx.x % WR_LANES;
  const uint32_t group = 0xFFFFu << (threadIdx.x & 16);
  for (Items it(Hkv); it.r < rows; it.next(Hkv)) {
    const int sl = slot[it.r], at = src ? src[it.r] : it.r;
    const bool in = at >= 0 && at < x.n_src;
    uint4 kx = make_uint4(0, 0, 0, 0), vx = kx;
    if (in) {  // the slot is not waited for
      const int q = x.one_seq ? 0 : at / x.n_per_seq, i = at - q * x.n_per_seq;
      const long long off = q * x.seq_stride + i * x.row_stride + it.h * x.head_stride;
      kx = reinterpret_cast<const uint4*>(x.k + off)[lane];
      vx = reinterpret_cast<const uint4*>(x.v + off)[lane];
    }
    if (!in || sl < 0 || sl >= n_slots) {  // the 16 lanes of a row agree
      if (sl >= 0 && lane == 0 && it.h == 0) fc_flag(FC_ERR_WORD(err), FC_EBIT_INVALID);
      continue;
    }
    auto top = [](const uint4& u) {
      const uint32_t m = __vmaxu2(__vmaxu2(u.x & 0x7FFF7FFFu, u.y & 0x7FFF7FFFu),
                                  __vmaxu2(u.z & 0x7FFF7FFFu, u.w & 0x7FFF7FFFu));
      return max(m & 0xFFFFu, m >> 16);
    };
    uint32_t m = top(kx) | (top(vx) << 16);
#pragma unroll
    for (int o = 1; o < WR_LANES; o <<= 1) m = __vmaxu2(m, __shfl_xor_sync(group, m, o));
    const long long row = ((long long)(sl >> shift) * Hkv + it.h) * (1 << shift) + (sl & ((1 << shift) - 1));
    auto scale = [](uint32_t bits) {
      return bits >= 0x7F80u ? __ushort_as_bfloat16(0x7FC0) : __float2bfloat16_rn(lo_f(bits) * (1.f / 7.f));
    };
    const __nv_bfloat16 sk = scale(m & 0xFFFFu), sv = scale(m >> 16);
    kc[row * WR_LANES + lane] = quantise8(kx, __bfloat162float(sk));
    vc[row * WR_LANES + lane] = quantise8(vx, __bfloat162float(sv));
    if (lane == 0) ks[row] = sk;
    if (lane == 1) vs[row] = sv;
  }
}

__global__ void __launch_bounds__(WR_THREADS, WR_CTAS) k_kv4_read(const int32_t* __restrict__ slot, int rows, int Hkv, int shift,
                                                         long long n_slots, const uint32_t* __restrict__ kc,
                                                         const uint32_t* __restrict__ vc,
                                                         const uint16_t* __restrict__ ks,
                                                         const uint16_t* __restrict__ vs, uint4* __restrict__ k,
                                                         uint4* __restrict__ v, unsigned int* err) {
  const int lane = threadIdx.x % WR_LANES;
  for (Items it(Hkv); it.r < rows; it.next(Hkv)) {
    const int sl = slot[it.r];
    if (sl >= n_slots && lane == 0 && it.h == 0) fc_flag(FC_ERR_WORD(err), FC_EBIT_INVALID);
    uint32_t a = 0x88888888u, b = a, sk = 0u, sv = 0u;  // zeros
    if (sl >= 0 && sl < n_slots) {
      const long long row = ((long long)(sl >> shift) * Hkv + it.h) * (1 << shift) + (sl & ((1 << shift) - 1));
      a = kc[row * WR_LANES + lane];
      b = vc[row * WR_LANES + lane];
      sk = ks[row];
      sv = vs[row];
    }
    // 0x4300 | c as bf16 is 128 + c: less 136 it is the number, exactly, and
    // times the scale the value, rounded once; in pairs (0, 4) (1, 5) ...
    auto values = [](uint32_t w, uint32_t s2) {
      uint32_t p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(p[i]) : "r"(((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u), "r"(0x43084308u));
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(p[i]) : "r"(p[i]), "r"(s2));
      }
      return make_uint4(__byte_perm(p[0], p[1], 0x5410), __byte_perm(p[2], p[3], 0x5410),
                        __byte_perm(p[0], p[1], 0x7632), __byte_perm(p[2], p[3], 0x7632));
    };
    const size_t to = ((size_t)it.r * Hkv + it.h) * WR_LANES + lane;
    __stcs(k + to, values(a, sk * 0x10001u));
    __stcs(v + to, values(b, sv * 0x10001u));
  }
}

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

unsigned grid_for(int rows, int Hkv) {
  // several times what is resident: CTAs that end early make room (16 an SM: 134 us, 64: 127 us)
  return (unsigned)std::min<long long>(((long long)rows * Hkv + WR_GROUPS - 1) / WR_GROUPS, 152 * 4 * WR_CTAS);
}

}  // namespace

fc_status fc_kv4_check(const fc_kv4_cache* c) {
  if (!c || c->n_pages < 1 || c->Hkv < 1) return FC_ERR_INVALID_ARG;
  if (c->D != HD || kv4_page_shift(c->page_size) < 0 || (long long)c->n_pages * c->page_size > 0x7FFFFFFFll)
    return FC_ERR_UNSUPPORTED;
  if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !aligned(c->k_codes, 16) ||
      !aligned(c->v_codes, 16) || !aligned(c->k_scale, 16) || !aligned(c->v_scale, 16))
    return FC_ERR_INVALID_ARG;
  return FC_OK;
}

extern "C" fc_status fc_kv_pages_plan(const int32_t* d_kv_len, const int32_t* d_n_new, int batch, int page_size,
                                      int32_t* d_table, int max_pages, const int32_t* d_free, int n_pages,
                                      const int32_t* d_n_free_in, const int32_t* d_path, int path_cap, int n_per_seq,
                                      int rows_cap, int32_t* d_cu, int32_t* d_seq, int32_t* d_pos, int32_t* d_slot,
                                      int32_t* d_src, int32_t* d_kv_len_out, int32_t* d_n_free_out,
                                      fc_stream stream) {
  FC_NVTX_RANGE();
  const int shift = kv4_page_shift(page_size);
  if (shift < 0) return FC_ERR_UNSUPPORTED;
  if (batch < 0 || max_pages < 1 || n_pages < 1 || rows_cap < 0 || (long long)n_pages << shift > 0x7FFFFFFFll)
    return FC_ERR_INVALID_ARG;
  if (batch == 0 && rows_cap == 0) return FC_OK;
  if ((batch && (!d_kv_len || !d_n_new || !d_table || !d_free || !d_kv_len_out)) || !d_n_free_in || !d_n_free_out ||
      !d_cu || d_n_free_in == d_n_free_out || (batch && d_kv_len == d_kv_len_out))
    return FC_ERR_INVALID_ARG;
  if (rows_cap && (!d_seq || !d_pos || !d_slot)) return FC_ERR_INVALID_ARG;
  if (d_src && (n_per_seq < 1 || (long long)batch * n_per_seq > 0x7FFFFFFFll || (d_path && path_cap < 1)))
    return FC_ERR_INVALID_ARG;
  PlanArgs a{d_kv_len, d_n_new,    batch,    shift,     max_pages, d_table, d_free, n_pages, d_n_free_in,
             d_path,   path_cap,   n_per_seq, rows_cap, d_cu,      d_seq,   d_pos,  d_slot,  d_src,
             d_kv_len_out, d_n_free_out, fc_error_slot()};
  int threads = 256;
  while (threads < PL_MAX_THREADS && threads < batch) threads *= 2;
  const int ctas = (int)std::max<long long>(
      1, std::min<long long>(((long long)rows_cap + threads * PL_ROWS - 1) / (threads * PL_ROWS), 152 * (2048 / threads)));
  const int per = (int)(((long long)rows_cap + ctas - 1) / ctas);
  k_pages_plan<<<ctas, threads, 0, static_cast<cudaStream_t>(stream)>>>(a, std::max(1, per));
  return FC_CHECK_LAUNCH();
}

extern "C" fc_status fc_kv_pages_release(const int32_t* d_kv_len, const int32_t* d_keep, int batch, int page_size,
                                         const int32_t* d_table, int max_pages, int32_t* d_free, int n_pages,
                                         const int32_t* d_n_free_in, int32_t* d_kv_len_out, int32_t* d_n_free_out,
                                         fc_stream stream) {
  FC_NVTX_RANGE();
  const int shift = kv4_page_shift(page_size);
  if (shift < 0) return FC_ERR_UNSUPPORTED;
  if (batch < 0 || max_pages < 1 || n_pages < 1) return FC_ERR_INVALID_ARG;
  if (batch == 0) return FC_OK;
  if (!d_kv_len || !d_keep || !d_table || !d_free || !d_n_free_in || !d_kv_len_out || !d_n_free_out ||
      d_n_free_in == d_n_free_out || d_kv_len == d_kv_len_out)
    return FC_ERR_INVALID_ARG;
  k_pages_release<<<1, PL_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(
      d_kv_len, d_keep, batch, shift, d_table, max_pages, d_free, n_pages, d_n_free_in, d_n_free_out, d_kv_len_out,
      fc_error_slot());
  return FC_CHECK_LAUNCH();
}

extern "C" fc_status fc_kv4_write(const fc_kv4_cache* cache, const void* d_k, const void* d_v, int n_seq, int n_per_seq,
                                  int64_t seq_stride, int64_t row_stride, int64_t head_stride, const int32_t* d_src,
                                  const int32_t* d_slot, int rows, fc_stream stream) {
  FC_NVTX_RANGE();
  if (const fc_status st = fc_kv4_check(cache)) return st;
  if (rows < 0 || n_seq < 0 || n_per_seq < 1 || seq_stride < 0 || row_stride < 0 || head_stride < 0 ||
      (long long)n_seq * n_per_seq > 0x7FFFFFFFll)
    return FC_ERR_INVALID_ARG;
  if (rows == 0) return FC_OK;
  if (!d_k || !d_v || !d_slot || !aligned(d_k, 16) || !aligned(d_v, 16) || seq_stride % 8 || row_stride % 8 ||
      head_stride % 8 || (!d_src && rows > n_seq * n_per_seq))
    return FC_ERR_INVALID_ARG;
  KvRows x{static_cast<const __nv_bfloat16*>(d_k), static_cast<const __nv_bfloat16*>(d_v), n_per_seq,
           n_seq * n_per_seq, n_seq == 1, seq_stride, row_stride, head_stride};
  if ((long long)rows * cache->Hkv > MAX_ITEMS) return FC_ERR_UNSUPPORTED;
  k_kv4_write<<<grid_for(rows, cache->Hkv), WR_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(
      x, d_src, d_slot, rows, cache->Hkv, kv4_page_shift(cache->page_size), (long long)cache->n_pages * cache->page_size,
      static_cast<uint32_t*>(cache->k_codes), static_cast<uint32_t*>(cache->v_codes),
      static_cast<__nv_bfloat16*>(cache->k_scale), static_cast<__nv_bfloat16*>(cache->v_scale), fc_error_slot());
  return FC_CHECK_LAUNCH();
}

extern "C" fc_status fc_kv4_read(const fc_kv4_cache* cache, const int32_t* d_slot, int rows, void* d_k, void* d_v,
                                 fc_stream stream) {
  FC_NVTX_RANGE();
  if (const fc_status st = fc_kv4_check(cache)) return st;
  if (rows < 0) return FC_ERR_INVALID_ARG;
  if (rows == 0) return FC_OK;
  if (!d_slot || !d_k || !d_v || !aligned(d_k, 16) || !aligned(d_v, 16)) return FC_ERR_INVALID_ARG;
  if ((long long)rows * cache->Hkv > MAX_ITEMS) return FC_ERR_UNSUPPORTED;
  k_kv4_read<<<grid_for(rows, cache->Hkv), WR_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(
      d_slot, rows, cache->Hkv, kv4_page_shift(cache->page_size), (long long)cache->n_pages * cache->page_size,
      static_cast<const uint32_t*>(cache->k_codes), static_cast<const uint32_t*>(cache->v_codes),
      static_cast<const uint16_t*>(cache->k_scale), static_cast<const uint16_t*>(cache->v_scale),
      static_cast<uint4*>(d_k), static_cast<uint4*>(d_v), fc_error_slot());
  return FC_CHECK_LAUNCH();
}
