// fc_kv8_evict: requests cut down to a number of cached tokens by the weights
// that attention gave them, every kv head choosing its own.
//
// For one request and head, of L tokens K stay: the tokens of the last `recent`
// positions, then those of the largest weight, ties to the lower index.  Those
// that stay at an index >= K (sources) move into the places below K that come
// free (holes), in order; a token below K that stays does not move.  So what is
// copied is what has to be, no source is a destination, and attention, which
// has no use for the order of keys, needs no table of its own.
//
//   k_select  a CTA a (request, head): the order of the tokens as 32-bit keys,
//             the K-th largest by three counts of 11, 11 and 10 bits (keys kept
//             in shared memory while they fit); who stays as a bit a token, whose
//             sums over groups of 32 rank ties, holes and sources without a walk;
//             then where every place's token comes from, its weight and position,
//             and a list of the blocks of 16 places that take a token.
//   k_move    a warp a block on the list: put together in registers (8 bytes a
//             lane of each row, lanes 0-15 keys, 16-31 values), it gets the scale
//             for what it then holds, below the old length (whose last block may
//             hold more than what stays); rows that change are written.  The block
//             that holds both the last places and the first sources is read from
//             a copy, as its own warp may have written it.
//
// Both are instructions and latency more than bytes: 32 requests of 8 heads and 4160
// tokens that lose 64 take 30 us (14 and 15), 16 requests of up to 16384 tokens that
// lose half 72 (15 and 56; 187 MB read, 110 written).
#include <algorithm>
#include <climits>

#include "kv8.cuh"

FC_DEFINE_ERROR_WORD(kv8_evict)

namespace {

constexpr int HD = KV8_D;
constexpr int SEL_THREADS = 1024;
constexpr int BINS = 2048;
constexpr int KEYS_SMEM = 40960;             // keys that fit in shared memory (160 KB)
constexpr int SEL_SMEM = KEYS_SMEM / 32 * 34 * 4;
constexpr int MAX_KEYS = SEL_SMEM / 8 * 32;  // 696,320 tokens a request
constexpr int MAX_RECENT = 1 << 22;
constexpr int MAX_CAP = 1 << 30;  // places of d_from are counted in 32 bits
constexpr uint32_t KEY_RECENT = 0xFF900000u;  // above every weight's key; recent tokens by age from here on
constexpr int MV_THREADS = 256, MV_WARPS = MV_THREADS / 32;
constexpr int EDGE_BYTES = 2 * KV8_BLOCK * HD + 16;  // a unit's copy: 16 rows of keys, of values, their scales

struct EvictArgs {
  const int32_t *table, *kv_len, *keep;
  int max_pages, n_pages, shift, Hkv, batch, cap, recent;
  const float* w_in;
  const int32_t* b_in;
  float* w_out;
  int32_t* b_out;
  int32_t* from;   // [batch][Hkv][cap]
  // workspace
  int32_t* count;       // [batch][Hkv] blocks on the list
  int32_t* todo;        // [batch][Hkv][ceil(cap / 16)] the list
  int32_t* list;        // [batch][Hkv][cap] sources in order, where they do not fit in shared memory
  unsigned char* edge;  // [batch][Hkv][EDGE_BYTES]
  uint8_t *kc, *vc;
  float *ks, *vs;
  unsigned int* err;
};

// A weight as an unsigned number of the same order: -0 like 0, NaN above infinity.
__device__ __forceinline__ uint32_t key_of(float w) {
  if (!(w == w)) return 0xFF800001u;
  const uint32_t u = __float_as_uint(w + 0.f);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// Inclusive sums over the block's threads, by way of one value a warp.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* s_sum) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, v, o);
    if (lane >= o) v += x;
  }
  __syncthreads();
  if (lane == 31) s_sum[warp] = v;
  __syncthreads();
  return v + __reduce_add_sync(0xFFFFFFFFu, lane < warp ? s_sum[lane] : 0u);
}

__device__ __forceinline__ uint32_t half2_bits(__half2 v) { return *reinterpret_cast<uint32_t*>(&v); }
__device__ __forceinline__ __half2 bits_half2(uint32_t v) { return *reinterpret_cast<__half2*>(&v); }

// A copy of the block that holds both places below keep and sources, by the block's threads.
__device__ __forceinline__ void copy_edge(const EvictArgs& a, int unit, int h, int keep, const int32_t* tab, int threads) {
  if (!(keep & (KV8_BLOCK - 1))) return;
  const int first = keep & ~(KV8_BLOCK - 1);
  const size_t p = ((((size_t)tab[first >> a.shift]) * a.Hkv + h) << a.shift) + (first & ((1 << a.shift) - 1));
  uint4* e = reinterpret_cast<uint4*>(a.edge + (size_t)unit * EDGE_BYTES);
  constexpr int N = KV8_BLOCK * HD / 16;
  for (int i = threadIdx.x; i < 2 * N; i += threads) e[i] = reinterpret_cast<const uint4*>((i < N ? a.kc : a.vc) + p * HD)[i % N];
  if (threadIdx.x < 2) reinterpret_cast<float*>(e + 2 * N)[threadIdx.x] = (threadIdx.x ? a.vs : a.ks)[p >> 4];
}

constexpr int HELD = 16;  // tokens a thread of k_select_held

// k_select for requests of up to HELD * THREADS tokens, whose weights and
// positions stay in registers from the first read on: only sources pass through
// shared memory.  Pages are looked up first, so that all reads are in flight at
// once.  (32 requests of 8 heads and 4160 tokens, caches flushed: 20 us, 23 with the
// pages looked up token by token, 25 with keys in shared memory and passes over them.)
template <int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_select_held(EvictArgs a) {
  constexpr int WARPS = THREADS / 32, GROUPS = HELD * WARPS, MOST = HELD * THREADS / 2;  // moves are at most half
  extern __shared__ uint32_t s_dyn[];
  int* s_src = reinterpret_cast<int*>(s_dyn);  // [MOST] sources: index, weight, position
  float* s_w = reinterpret_cast<float*>(s_dyn + MOST);
  int* s_b = reinterpret_cast<int*>(s_dyn + 2 * MOST);
  __shared__ __align__(16) uint32_t s_hist[BINS];
  __shared__ uint32_t s_sum[32], s_bits[GROUPS], s_tie[GROUPS], s_rank[GROUPS], s_page[THREADS];  // (pages of 16 tokens and more)
  __shared__ int s_newest, s_todo;
  __shared__ uint32_t s_digit, s_left, s_in_bin;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.x, b = unit / a.Hkv, h = unit - b * a.Hkv;
  const int L = a.kv_len[b], keep = a.keep[b];
  const int32_t* tab = a.table + (size_t)b * a.max_pages;
  int32_t* from = a.from + (size_t)unit * a.cap;
  const bool wrong = L < 0 || keep < 0 || L > (long long)a.max_pages << a.shift;
  const bool full = !wrong && keep < L && keep > a.cap;
  if (tid == 0) s_newest = INT_MIN, s_todo = 0;
  for (int i = tid; i < BINS; i += THREADS) s_hist[i] = 0;
  const bool fine = !wrong && !full;
  const int pages = fine ? (L + (1 << a.shift) - 1) >> a.shift : 0;  // at most THREADS
  bool bad = false;
  if (tid < pages) {
    const int page = tab[tid];
    s_page[tid] = ((uint32_t)page * (uint32_t)a.Hkv + (uint32_t)h) << a.shift;  // its first place
    bad = (uint32_t)page >= (uint32_t)a.n_pages;
  }
  const bool ok = !__syncthreads_or(bad) && fine;
  auto at = [&](int i) { return s_page[i >> a.shift] | ((uint32_t)i & ((1u << a.shift) - 1u)); };
  float w[HELD];
  int born[HELD];
#pragma unroll
  for (int u = 0; u < HELD; ++u) {
    const int i = u * THREADS + tid;
    const bool in = ok && i < L;
    const uint32_t p = in ? at(i) : 0u;
    w[u] = in ? __ldg(a.w_in + p) : 0.f;
    born[u] = in ? __ldg(a.b_in + p) : INT_MIN;
  }
  if (!ok) {  // left as it is
    if (tid == 0) {
      a.count[unit] = 0;
      if (h == 0) fc_flag(FC_ERR_WORD(a.err), full ? FC_EBIT_CAPACITY : FC_EBIT_INVALID);
    }
    for (int i = tid; i < a.cap; i += THREADS) from[i] = -1;
    return;
  }
  if (a.recent > 0) {
    int newest = INT_MIN;
#pragma unroll
    for (int u = 0; u < HELD; ++u) newest = max(newest, born[u]);
    newest = __reduce_max_sync(0xFFFFFFFFu, newest);
    if (lane == 0) atomicMax(&s_newest, newest);
  }
  __syncthreads();
  const bool lose = keep < L;
  const int kept = min(keep, L);
  uint32_t below = (1u << lane) - 1u;
  auto lows = [&](int g) { return kept <= 32 * g ? 0u : kept - 32 * g >= 32 ? 0xFFFFFFFFu : (1u << (kept - 32 * g)) - 1u; };
  uint32_t stays = 0;  // bit u: token u * THREADS + tid does
  if (lose && keep > 0) {
    const long long after = (long long)s_newest - a.recent;  // positions above this are recent
    uint32_t key[HELD];
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
      const long long age = (long long)born[u] - after;
      key[u] = a.recent > 0 && age > 0 ? KEY_RECENT + (uint32_t)age : key_of(w[u]);
    }
    uint32_t prefix = 0, mask = 0, want = (uint32_t)keep;  // keys of this prefix still wanted
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int low = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t digits = pass == 2 ? 1023u : 2047u;
#pragma unroll
      for (int u = 0; u < HELD; ++u) {
        if (u * THREADS >= L) break;
        const bool in = u * THREADS + tid < L && (key[u] & mask) == prefix;
        if (pass > 0 && !__any_sync(0xFFFFFFFFu, in)) continue;
        const uint32_t digit = in ? (key[u] >> low) & digits : BINS;
        // many tokens may have one weight, 0 above all: a warp of them is one addition
        const uint32_t first = __shfl_sync(0xFFFFFFFFu, digit, 0);
        if (__all_sync(0xFFFFFFFFu, digit == first)) {
          if (lane == 0 && first < BINS) atomicAdd(&s_hist[first], 32u);
        } else if (digit < BINS) {
          atomicAdd(&s_hist[digit], 1u);
        }
      }
      __syncthreads();
      // the bin where the count from above reaches `want`: some bins a thread, from the top
      constexpr int EACH = BINS / THREADS;
      const int top = BINS - 1 - EACH * tid;
      uint32_t c[EACH], sum = 0;
#pragma unroll
      for (int j = 0; j < EACH; ++j) sum += c[j] = s_hist[top - j];
      uint32_t above = block_scan(sum, s_sum) - sum;
#pragma unroll
      for (int j = 0; j < EACH; ++j) {
        if (above < want && want <= above + c[j]) s_digit = top - j, s_left = want - above, s_in_bin = c[j];
        above += c[j];
        s_hist[top - j] = 0;
      }
      __syncthreads();
      prefix |= s_digit << low;
      mask |= digits << low;
      want = s_left;
      if (want == s_in_bin) break;  // all of the bin's keys stay: the rest of the bits do not matter
    }
    const bool all_ties = want == s_in_bin;
    uint32_t ties = 0;
#pragma unroll
    for (int u = 0; u < HELD; ++u) {
      if (u * THREADS >= L) break;
      const bool in = u * THREADS + tid < L;
      const uint32_t k = key[u] & mask;
      if (in && (all_ties ? k >= prefix : k > prefix)) stays |= 1u << u;
      if (!all_ties) {
        const bool tie = in && k == prefix;
        const uint32_t m = __ballot_sync(0xFFFFFFFFu, tie);
        if (tie) ties |= 1u << u;
        if (lane == 0) s_tie[u * WARPS + warp] = m;
      }
    }
    if (!all_ties) {  // the first `want` of the ties stay
      __syncthreads();
      const uint32_t c = tid < GROUPS && 32 * tid < L ? __popc(s_tie[tid]) : 0u;
      const uint32_t rank = block_scan(c, s_sum) - c;
      if (tid < GROUPS) s_rank[tid] = rank;
      __syncthreads();
#pragma unroll
      for (int u = 0; u < HELD; ++u) {
        const int g = u * WARPS + warp;
        if ((ties >> u) & 1u)
          if (s_rank[g] + __popc(s_tie[g] & below) < want) stays |= 1u << u;
      }
      __syncthreads();
    }
  } else if (!lose) {
    stays = 0xFFFFFFFFu;
  }
  // ---- ranks of holes (low half) and sources (high half), a group of 32 a thread
#pragma unroll
  for (int u = 0; u < HELD; ++u) {
    if (u * THREADS >= L) break;
    const uint32_t m = __ballot_sync(0xFFFFFFFFu, u * THREADS + tid < L && ((stays >> u) & 1u));
    if (lane == 0) s_bits[u * WARPS + warp] = m;
  }
  __syncthreads();
  if (lose) {
    uint32_t c = 0;
    if (tid < GROUPS && 32 * tid < L) {
      const uint32_t s = s_bits[tid], lo = lows(tid);
      c = __popc(~s & lo) | ((uint32_t)__popc(s & ~lo) << 16);
    }
    const uint32_t rank = block_scan(c, s_sum) - c;
    if (tid < GROUPS) s_rank[tid] = rank;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < HELD; ++u) {  // the sources, in order
      const int i = u * THREADS + tid, g = u * WARPS + warp;
      if (i >= keep && i < L && ((stays >> u) & 1u)) {
        const uint32_t r = (s_rank[g] >> 16) + __popc(s_bits[g] & ~lows(g) & below);
        s_src[r] = i;
        s_w[r] = w[u];
        s_b[r] = born[u];
      }
    }
    // the blocks that take a token
    int32_t* todo = a.todo + (size_t)unit * ((a.cap + KV8_BLOCK - 1) / KV8_BLOCK);
    const int blocks = (keep + KV8_BLOCK - 1) / KV8_BLOCK;
    for (int t0 = 32 * warp; t0 < blocks; t0 += THREADS) {
      const int t = t0 + lane;
      const bool takes = t < blocks && (((~s_bits[t >> 1] & lows(t >> 1)) >> (16 * (t & 1))) & 0xFFFFu);
      const uint32_t all = __ballot_sync(0xFFFFFFFFu, takes);
      int at0 = 0;
      if (lane == 0 && all) at0 = atomicAdd(&s_todo, __popc(all));
      at0 = __shfl_sync(0xFFFFFFFFu, at0, 0);
      if (takes) todo[at0 + __popc(all & below)] = t;
    }
    copy_edge(a, unit, h, keep, tab, THREADS);
  }
  __syncthreads();
  if (tid == 0) a.count[unit] = s_todo;
#pragma unroll
  for (int u = 0; u < HELD; ++u) {
    const int i = u * THREADS + tid, g = u * WARPS + warp;
    if (i >= kept) break;
    const uint32_t gone = lose ? ~s_bits[g] & lows(g) : 0u;
    int src = -1;
    if ((gone >> lane) & 1u) {
      const uint32_t r = (s_rank[g] & 0xFFFFu) + __popc(gone & below);
      src = s_src[r];
      w[u] = s_w[r];
      born[u] = s_b[r];
    }
    const uint32_t p = at(i);
    a.w_out[p] = w[u];
    a.b_out[p] = born[u];
    if (i < a.cap) from[i] = src;
  }
  for (int i = kept + tid; i < a.cap; i += THREADS) from[i] = -1;
}

// Threads: a power of two, 512 to SEL_THREADS.  Shared memory: held_cap keys (the
// sources' list takes their place) and two words a group of 32 tokens, or, of a
// longer request, these words alone.
__global__ void __launch_bounds__(SEL_THREADS) k_select(EvictArgs a, int held_cap) {
  extern __shared__ uint32_t s_dyn[];
  __shared__ uint32_t s_hist[BINS];
  __shared__ uint32_t s_sum[32];
  __shared__ int s_bad, s_newest, s_todo;
  __shared__ uint32_t s_digit, s_left, s_in_bin;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  const int unit = blockIdx.x, b = unit / a.Hkv, h = unit - b * a.Hkv;
  const int L = a.kv_len[b], keep = a.keep[b];
  const int32_t* tab = a.table + (size_t)b * a.max_pages;
  int32_t* from = a.from + (size_t)unit * a.cap;
  const bool wrong = L < 0 || keep < 0 || L > (long long)a.max_pages << a.shift;
  const bool full = !wrong && keep < L && keep > a.cap;
  const bool held = L <= held_cap;
  uint32_t* s_keys = s_dyn;
  uint32_t* bits = held ? s_dyn + held_cap : s_dyn;
  int32_t* list = held ? reinterpret_cast<int32_t*>(s_keys) : a.list + (size_t)unit * a.cap;
  if (tid == 0) s_bad = 0, s_newest = INT_MIN, s_todo = 0;
  for (int i = tid; i < BINS; i += threads) s_hist[i] = 0;
  __syncthreads();
  // a token's place; false for a page outside the pool
  auto at = [&](int i, uint32_t& p) {
    const uint32_t page = (uint32_t)__ldg(tab + (i >> a.shift));
    p = ((page * (uint32_t)a.Hkv + (uint32_t)h) << a.shift) | ((uint32_t)i & ((1u << a.shift) - 1u));
    return page < (uint32_t)a.n_pages;
  };
  const bool lose = !wrong && !full && keep < L;
  // weights and positions of places 0 .. n - 1, from the indexes that `source` gives; four loads ahead of their stores
  auto copy_tracks = [&](int n, auto&& source) {
    for (int i0 = tid; i0 < n; i0 += 4 * threads) {
      uint32_t p[4];
      float w[4];
      int born[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u * threads;
        if (i >= n) continue;
        uint32_t q;
        at(i, p[u]);
        at(source(i), q);
        w[u] = __ldg(a.w_in + q);
        born[u] = __ldg(a.b_in + q);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i0 + u * threads < n) a.w_out[p[u]] = w[u], a.b_out[p[u]] = born[u];
    }
  };
  if (!wrong && !full) {
    int newest = INT_MIN;
    bool bad = false;
    const bool read_born = lose && a.recent > 0, read_weight = lose && held;
#pragma unroll 4
    for (int i = tid; i < L; i += threads) {
      uint32_t p;
      const bool ok = at(i, p);
      bad |= !ok;
      const int born = ok && read_born ? __ldg(a.b_in + p) : INT_MIN;
      const float weight = ok && read_weight ? __ldg(a.w_in + p) : 0.f;
      newest = max(newest, born);
      if (read_weight) s_keys[i] = key_of(weight);
    }
    if (bad) s_bad = 1;
    newest = __reduce_max_sync(0xFFFFFFFFu, newest);
    if (lane == 0 && newest != INT_MIN) atomicMax(&s_newest, newest);
  }
  __syncthreads();
  if (wrong || full || s_bad) {  // left as it is
    if (tid == 0) {
      a.count[unit] = 0;
      if (h == 0) fc_flag(FC_ERR_WORD(a.err), full ? FC_EBIT_CAPACITY : FC_EBIT_INVALID);
    }
    for (int i = tid; i < a.cap; i += threads) from[i] = -1;
    return;
  }
  if (!lose) {
    if (tid == 0) a.count[unit] = 0;
    for (int i = tid; i < a.cap; i += threads) from[i] = -1;
    copy_tracks(L, [&](int i) { return i; });
    return;
  }
  // ---- keys, the first count with them
  const long long after = (long long)s_newest - a.recent;  // positions above this are recent
  auto make_key = [&](int i, bool have) {
    uint32_t p;
    if (a.recent > 0 || !have) at(i, p);
    if (a.recent > 0) {
      const long long age = (long long)__ldg(a.b_in + p) - after;
      if (age > 0) return KEY_RECENT + (uint32_t)age;
    }
    return have ? s_keys[i] : key_of(__ldg(a.w_in + p));
  };
  auto key = [&](int i) { return held ? s_keys[i] : make_key(i, false); };
  uint32_t prefix = 0, mask = 0, want = (uint32_t)keep;  // keys of this prefix still wanted
#pragma unroll 1
  for (int pass = 0; pass < 3 && keep > 0; ++pass) {
    const int low = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
    auto count = [&](bool in, uint32_t k) {
      const uint32_t digit = in && (k & mask) == prefix ? (k >> low) & ((1u << width) - 1u) : BINS;
      // many tokens may have one weight, 0 above all: a warp of them is one addition
      const uint32_t first = __shfl_sync(0xFFFFFFFFu, digit, 0);
      if (__all_sync(0xFFFFFFFFu, digit == first)) {
        if (lane == 0 && first < BINS) atomicAdd(&s_hist[first], 32u);
      } else if (digit < BINS) {
        atomicAdd(&s_hist[digit], 1u);
      }
    };
    if (pass == 0 && held) {
#pragma unroll 4
      for (int i0 = 32 * warp; i0 < L; i0 += threads) {
        const int i = i0 + lane;
        const uint32_t k = i < L ? make_key(i, true) : 0u;
        if (i < L) s_keys[i] = k;
        count(i < L, k);
      }
    } else {
      for (int i0 = 32 * warp; i0 < L; i0 += threads) count(i0 + lane < L, i0 + lane < L ? key(i0 + lane) : 0u);
    }
    __syncthreads();
    // the bin where the count from above reaches `want`: some bins a thread, from the top
    const int each = BINS / threads, top = BINS - 1 - each * tid;
    uint32_t sum = 0;
    for (int j = 0; j < each; ++j) sum += s_hist[top - j];
    uint32_t above = block_scan(sum, s_sum) - sum;
    for (int j = 0; j < each; ++j) {
      const uint32_t c = s_hist[top - j];
      if (above < want && want <= above + c) s_digit = top - j, s_left = want - above, s_in_bin = c;
      above += c;
      s_hist[top - j] = 0;
    }
    __syncthreads();
    prefix |= s_digit << low;
    mask |= ((1u << width) - 1u) << low;
    want = s_left;
    // all of the bin's keys stay: the rest of the bits do not matter
    if (want == s_in_bin) break;
  }
  // keys whose masked bits are above prefix stay, and the first `want` of those equal to it (all, if there are no more)
  const bool all_ties = keep > 0 && want == s_in_bin;
  const int groups = (L + 31) >> 5;
  for (int g = warp; g < groups; g += warps) {
    const int i = 32 * g + lane;
    const uint32_t k = i < L && keep > 0 ? key(i) & mask : 0u;
    const uint32_t up = __ballot_sync(0xFFFFFFFFu, i < L && keep > 0 && (all_ties ? k >= prefix : k > prefix));
    const uint32_t tie = __ballot_sync(0xFFFFFFFFu, i < L && keep > 0 && k == prefix);
    if (lane == 0) {
      bits[2 * g] = up;
      if (!all_ties) bits[2 * g + 1] = tie;
    }
  }
  __syncthreads();
  const int each = (groups + threads - 1) / threads, g0 = min(groups, tid * each), g1 = min(groups, g0 + each);
  if (!all_ties && keep > 0) {
    uint32_t n = 0;
    for (int g = g0; g < g1; ++g) n += __popc(bits[2 * g + 1]);
    uint32_t rank = block_scan(n, s_sum) - n;
    for (int g = g0; g < g1; ++g) {
      uint32_t tie = bits[2 * g + 1];
      const uint32_t c = __popc(tie), room = want > rank ? want - rank : 0u;
      for (uint32_t x = room; x < c; ++x) tie &= ~(0x80000000u >> __clz(tie));  // the last ones go
      bits[2 * g] |= tie;
      rank += c;
    }
  }
  // ---- holes (bits 0..15 of a sum) and sources; at most 2^31 tokens, so a sum each
  auto lows = [&](int g) { return keep <= 32 * g ? 0u : keep - 32 * g >= 32 ? 0xFFFFFFFFu : (1u << (keep - 32 * g)) - 1u; };
  uint32_t nh = 0, ns = 0;
  for (int g = g0; g < g1; ++g) {
    const uint32_t s = bits[2 * g], lo = lows(g);
    nh += __popc(~s & lo);
    ns += __popc(s & ~lo);
  }
  nh = block_scan(nh, s_sum) - nh;
  ns = block_scan(ns, s_sum) - ns;
  for (int g = g0; g < g1; ++g) {  // a group's second word: its first hole's or source's rank (of the group with both, the hole's)
    const uint32_t s = bits[2 * g], lo = lows(g);
    bits[2 * g + 1] = lo ? nh : ns;
    for (uint32_t m = lo ? s & ~lo : 0u, r = ns; m; m &= m - 1, ++r) list[r] = 32 * g + __ffs(m) - 1;
    nh += __popc(~s & lo);
    ns += __popc(s & ~lo);
  }
  __syncthreads();
  const uint32_t below = (1u << lane) - 1u;
  for (int g = (keep + 31) / 32 + warp; g < groups; g += warps) {  // the sources, in order
    const uint32_t s = bits[2 * g];
    if ((s >> lane) & 1u) list[bits[2 * g + 1] + __popc(s & below)] = 32 * g + lane;
  }
  // ---- the blocks that take a token
  int32_t* todo = a.todo + (size_t)unit * ((a.cap + KV8_BLOCK - 1) / KV8_BLOCK);
  for (int t0 = 32 * warp; t0 < (keep + KV8_BLOCK - 1) / KV8_BLOCK; t0 += threads) {
    const int t = t0 + lane;
    const bool takes = t < (keep + KV8_BLOCK - 1) / KV8_BLOCK && (((~bits[t & ~1] & lows(t >> 1)) >> (16 * (t & 1))) & 0xFFFFu);
    const uint32_t all = __ballot_sync(0xFFFFFFFFu, takes);
    int at0 = 0;
    if (lane == 0 && all) at0 = atomicAdd(&s_todo, __popc(all));
    at0 = __shfl_sync(0xFFFFFFFFu, at0, 0);
    if (takes) todo[at0 + __popc(all & below)] = t;
  }
  copy_edge(a, unit, h, keep, tab, threads);
  __syncthreads();
  if (tid == 0) a.count[unit] = s_todo;
  copy_tracks(keep, [&](int i) {
    const int g = i >> 5;
    const uint32_t gone = ~bits[2 * g] & lows(g);
    const bool hole = (gone >> (i & 31)) & 1u;
    const int src = hole ? list[bits[2 * g + 1] + __popc(gone & ((1u << (i & 31)) - 1u))] : -1;
    from[i] = src;
    return hole ? src : i;
  });
  for (int i = keep + tid; i < a.cap; i += threads) from[i] = -1;
}

// Registers bound how many blocks are in flight (5 CTAs an SM at 48: half of 16 x
// 16384 tokens 72 us, 4 81, 6 with spills 82), instructions what a block takes.
__global__ void __launch_bounds__(MV_THREADS, 5) k_move(EvictArgs a) {
  const int lane = threadIdx.x & 31, l16 = lane & 15, half = (threadIdx.x >> 5) & 1;
  const int unit = blockIdx.x, n = a.count[unit];
  const int b = unit / a.Hkv, h = unit - b * a.Hkv;
  const int keep = a.keep[b], L = a.kv_len[b];
  const int32_t* from = a.from + (size_t)unit * a.cap;
  const int32_t* todo = a.todo + (size_t)unit * ((a.cap + KV8_BLOCK - 1) / KV8_BLOCK);
  const int32_t* tab = a.table + (size_t)b * a.max_pages;
  const unsigned char* edge = a.edge + (size_t)unit * EDGE_BYTES;
  auto at = [&](int i) { return (((uint32_t)tab[i >> a.shift] * (uint32_t)a.Hkv + (uint32_t)h) << a.shift) | ((uint32_t)i & ((1u << a.shift) - 1u)); };
  uint8_t* codes = half ? a.vc : a.kc;
  float* scales = half ? a.vs : a.ks;
  // a block's number and where its rows come from are asked for one block ahead
  const int step = gridDim.y * (MV_WARPS / 2);
  auto source = [&](int base) { return l16 + base < keep ? from[base + l16] : -1; };
  int x = blockIdx.y * (MV_WARPS / 2) + (threadIdx.x >> 6);
  int base_next = x < n ? todo[x] * KV8_BLOCK : 0, mine_next = x < n ? source(base_next) : -1;
#pragma unroll 1
  for (; x < n; x += step) {
    const int base = base_next, mine = mine_next, live = min(KV8_BLOCK, L - base);
    if (x + step < n) base_next = todo[x + step] * KV8_BLOCK;
    const uint32_t to = at(base);
    // lane l16: where row l16 is, and its scale
    const bool copied = mine >= 0 && (keep & (KV8_BLOCK - 1)) && mine >> 4 == keep >> 4;
    const uint32_t row = mine >= 0 && !copied ? at(mine) : to + l16;
    const float row_scale = copied ? reinterpret_cast<const float*>(edge + 2 * KV8_BLOCK * HD)[half] : scales[row >> 4];
    const uint32_t moved = __ballot_sync(0xFFFFFFFFu, mine >= 0), copies = __ballot_sync(0xFFFFFFFFu, copied);
    const uint32_t* at_lane = reinterpret_cast<const uint32_t*>(codes) + lane;
    uint32_t w[KV8_BLOCK];
#pragma unroll
    for (int j = 0; j < KV8_BLOCK; ++j) w[j] = at_lane[(size_t)__shfl_sync(0xFFFFFFFFu, row, j) * (HD / 4)];
    if (copies) {
#pragma unroll
      for (int j = 0; j < KV8_BLOCK; ++j) {
        const int k = __shfl_sync(0xFFFFFFFFu, mine, j) & 15;
        if ((copies >> j) & 1u) w[j] = reinterpret_cast<const uint32_t*>(edge + (half * KV8_BLOCK + k) * HD)[lane];
      }
    }
    if (x + step < n) mine_next = source(base_next);
    // The largest magnitude: the seven bits of a number's are 8 E + m, of (1 + m / 8) 2^(E - 7) from 8 on, so
    // that 2^-d times it has them less 8 d.  (Below 8, subnormal, it is less than that says: none of these is
    // the largest beside one of 8 or more.)  Two in 16 bits each, 0x4000 added.
    const bool nan = __any_sync(0xFFFFFFFFu, l16 < live && kv8_nan(row_scale));
    const int row_e = l16 < live ? min(max(kv8_exp(row_scale), KV8_MIN_EXP), KV8_MAX_EXP) : KV8_MIN_EXP;
    const int ref = __reduce_max_sync(0xFFFFFFFFu, row_e);
    const uint32_t bias = l16 < live ? 0x40004000u - (uint32_t)(ref - row_e) * 0x00080008u : 0u;
    uint32_t top2 = 0;
#pragma unroll
    for (int j = 0; j < KV8_BLOCK; ++j)
      top2 = __vmaxu2(top2, __vmaxu2(w[j] & 0x007F007Fu, (w[j] >> 8) & 0x007F007Fu) + __shfl_sync(0xFFFFFFFFu, bias, j));
    const int bits = (int)__reduce_max_sync(0xFFFFFFFFu, max(top2 & 0xFFFFu, top2 >> 16)) - 0x4000;
    int e;  // the smallest with (1 + m / 8) 2^(E - 7) 2^ref <= 1.75 * 2^(e + 8)
    if (bits >= 8) {
      e = max(ref + (bits >> 3) - 15 + ((bits & 7) == 7 ? 1 : 0), KV8_MIN_EXP);
    } else {  // from the numbers themselves, times 2^-6 so that none overflows
      float top = 0.f;
#pragma unroll
      for (int j = 0; j < KV8_BLOCK; ++j) {
        const float s = kv8_pow2(__shfl_sync(0xFFFFFFFFu, row_e, j) - 6);
        const float2 p = e4m3x2_floats(w[j] & 0xFFFFu), q = e4m3x2_floats(w[j] >> 16);
        if (j < live) top = fmaxf(top, fmaxf(fmaxf(fabsf(p.x), fabsf(p.y)), fmaxf(fabsf(q.x), fabsf(q.y))) * s);
      }
      top = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top)));
      e = max(kv8_exp_for(top) + 6, KV8_MIN_EXP);
    }
    const int d = nan ? 0 : row_e - e;
    const uint32_t by = half2_bits(kv8_half_pow2(d));
    const uint32_t again = __ballot_sync(0xFFFFFFFFu, d != 0);                // rows of another scale, rounded again
    const uint32_t put = (moved | again) & ((1u << live) - 1u);  // rows that change
    const bool large = __any_sync(0xFFFFFFFFu, l16 < live && d > 15);
    uint32_t* out = reinterpret_cast<uint32_t*>(codes + (size_t)to * HD) + lane;
#pragma unroll
    for (int j = 0; j < KV8_BLOCK; ++j) {
      if (!((put >> j) & 1u)) continue;
      uint32_t r = w[j];
      if ((again >> j) & 1u) r = large ? kv8_rescale4(r, __shfl_sync(0xFFFFFFFFu, d, j)) : kv8_times4(r, bits_half2(__shfl_sync(0xFFFFFFFFu, by, j)));
      out[j * 32] = r;
    }
    if (lane == 0) scales[to >> 4] = nan ? __uint_as_float(0x7FC00000u) : kv8_pow2(e);
  }
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

extern "C" size_t fc_kv8_evict_workspace(int batch, int Hkv, int cap) {
  if (batch < 1 || Hkv < 1 || cap < 0 || cap > MAX_CAP) return 0;
  const size_t units = (size_t)batch * Hkv;
  return up256(units * 4) + up256(units * ((cap + KV8_BLOCK - 1) / KV8_BLOCK) * 4) + up256(units * EDGE_BYTES) + up256(units * cap * 4);
}

extern "C" fc_status fc_kv8_evict(const fc_kv8_cache* cache, const int32_t* d_table, int max_pages, const int32_t* d_kv_len,
                                  const int32_t* d_keep, int batch, int recent, const float* d_weight_in,
                                  const int32_t* d_born_in, float* d_weight_out, int32_t* d_born_out, int32_t* d_from, int cap,
                                  void* d_ws, size_t ws_bytes, fc_stream stream) {
  FC_NVTX_RANGE();
  if (const fc_status st = fc_kv8_check(cache)) return st;
  const int shift = kv8_page_shift(cache->page_size);
  if (batch < 0 || max_pages < 1 || recent < 0 || cap < 0) return FC_ERR_INVALID_ARG;
  if (recent > MAX_RECENT || cap > MAX_CAP || (long long)max_pages << shift > MAX_KEYS || (long long)batch * cache->Hkv > 1 << 24)
    return FC_ERR_UNSUPPORTED;
  if (batch == 0) return FC_OK;
  if (!d_table || !d_kv_len || !d_keep || !d_weight_in || !d_born_in || !d_weight_out || !d_born_out || (cap && !d_from) ||
      d_weight_in == d_weight_out || d_born_in == d_born_out)
    return FC_ERR_INVALID_ARG;
  const long long units = (long long)batch * cache->Hkv, longest = (long long)max_pages << shift;
  if (!d_ws || !kv8_aligned(d_ws, 256) || ws_bytes < fc_kv8_evict_workspace(batch, cache->Hkv, cap)) return FC_ERR_WORKSPACE;
  unsigned char* ws = static_cast<unsigned char*>(d_ws);
  auto take = [&](size_t n) {
    unsigned char* p = ws;
    ws += up256(n);
    return p;
  };
  const int blocks = (cap + KV8_BLOCK - 1) / KV8_BLOCK;
  EvictArgs a{d_table, d_kv_len, d_keep, max_pages, cache->n_pages, shift, cache->Hkv, batch, cap, recent, d_weight_in, d_born_in,
              d_weight_out, d_born_out, d_from, nullptr, nullptr, nullptr, nullptr,
              static_cast<uint8_t*>(cache->k_codes), static_cast<uint8_t*>(cache->v_codes), static_cast<float*>(cache->k_scale),
              static_cast<float*>(cache->v_scale), fc_error_slot()};
  a.count = reinterpret_cast<int32_t*>(take(units * 4));
  a.todo = reinterpret_cast<int32_t*>(take(units * blocks * 4));
  a.edge = take(units * EDGE_BYTES);
  a.list = reinterpret_cast<int32_t*>(take(units * cap * 4));
  static std::atomic<unsigned long long> done{0};
  const fc_status st = fc_once_per_device(done, [](int) {
    if (cudaFuncSetAttribute(k_select_held<512>, cudaFuncAttributeMaxDynamicSharedMemorySize, HELD * 512 / 2 * 12) != cudaSuccess ||
        cudaFuncSetAttribute(k_select_held<1024>, cudaFuncAttributeMaxDynamicSharedMemorySize, HELD * 1024 / 2 * 12) != cudaSuccess)
      return FC_ERR_CUDA;
    return fc_cuda_status(cudaFuncSetAttribute(k_select, cudaFuncAttributeMaxDynamicSharedMemorySize, SEL_SMEM));
  });
  if (st != FC_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int held = (int)std::min<long long>((longest + 31) / 32 * 32, KEYS_SMEM);
  if (longest <= HELD * 256) k_select_held<256><<<(unsigned)units, 256, HELD * 256 / 2 * 12, s>>>(a);
  else if (longest <= HELD * 512) k_select_held<512><<<(unsigned)units, 512, HELD * 512 / 2 * 12, s>>>(a);
  else if (longest <= HELD * 1024) k_select_held<1024><<<(unsigned)units, 1024, HELD * 1024 / 2 * 12, s>>>(a);
  else k_select<<<(unsigned)units, SEL_THREADS, longest > KEYS_SMEM ? SEL_SMEM : held / 32 * 34 * 4, s>>>(a, held);
  if (cap > 0) {
    // CTAs a unit: enough for every SM's registers, while there are blocks for them
    const int y = (int)std::max<long long>(1, std::min<long long>((152 * 20 + units - 1) / units, (2 * blocks + MV_WARPS - 1) / MV_WARPS));
    k_move<<<dim3((unsigned)units, (unsigned)y), MV_THREADS, 0, s>>>(a);
  }
  return FC_CHECK_LAUNCH();
}
