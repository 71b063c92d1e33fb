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
//             in shared memory while they fit), then warps that each own a run
//             of indexes count ties, holes and sources, and write where every
//             place's token comes from, its weight and its position.
//   k_move    a warp a block of 16 places: one that takes a token is put
//             together in registers (8 bytes a lane of each row, lanes 0-15 keys, 16-31
//             values), gets the scale for what it then holds and is written
//             whole.  The block that holds both the last places and the first
//             sources changes its scale too, so it is left for a second launch.
#include <algorithm>
#include <climits>

#include "kv8.cuh"

FC_DEFINE_ERROR_WORD(kv8_evict)

namespace {

constexpr int HD = KV8_D;
constexpr int SEL_THREADS = 1024, SEL_WARPS = SEL_THREADS / 32;
constexpr int BINS = 2048;
constexpr int KEYS_SMEM = 49152;             // keys that fit in shared memory (192 KB)
constexpr int MAX_RECENT = 1 << 22;
constexpr uint32_t KEY_RECENT = 0xFF900000u;  // above every weight's key; recent tokens by age from here on
constexpr int MV_THREADS = 256, MV_WARPS = MV_THREADS / 32;

struct EvictArgs {
  const int32_t *table, *kv_len, *keep;
  int max_pages, n_pages, shift, Hkv, batch, cap, recent;
  const float* w_in;
  const int32_t* b_in;
  float* w_out;
  int32_t* b_out;
  int32_t* from;   // [batch][Hkv][cap]
  int32_t* list;   // workspace [batch][Hkv][cap]: sources in order
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

__global__ void __launch_bounds__(SEL_THREADS) k_select(EvictArgs a) {
  extern __shared__ uint32_t s_keys[];
  __shared__ uint32_t s_hist[BINS];
  __shared__ int s_warp[SEL_WARPS][3];
  __shared__ uint32_t s_sum[SEL_WARPS];
  __shared__ int s_bad, s_newest;
  __shared__ uint32_t s_digit, s_left;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.x, b = unit / a.Hkv, h = unit - b * a.Hkv;
  int L = a.kv_len[b], keep = a.keep[b];
  const int32_t* tab = a.table + (size_t)b * a.max_pages;
  int32_t* from = a.from + (size_t)unit * a.cap;
  int32_t* list = a.list + (size_t)unit * a.cap;
  if (tid == 0) s_bad = 0, s_newest = INT_MIN;
  __syncthreads();
  const bool wrong = L < 0 || keep < 0 || L > (long long)a.max_pages << a.shift;
  if (!wrong)
    for (int i = tid; i < (int)(((long long)L + (1 << a.shift) - 1) >> a.shift); i += SEL_THREADS)
      if ((unsigned)tab[i] >= (unsigned)a.n_pages) s_bad = 1;
  __syncthreads();
  const bool full = !wrong && keep < L && keep > a.cap;
  if (wrong || s_bad || full) {  // left as it is
    if (tid == 0 && h == 0) fc_flag(FC_ERR_WORD(a.err), full && !s_bad ? FC_EBIT_CAPACITY : FC_EBIT_INVALID);
    for (int i = tid; i < a.cap; i += SEL_THREADS) from[i] = -1;
    return;
  }
  auto at = [&](int i) { return ((((size_t)tab[i >> a.shift]) * a.Hkv + h) << a.shift) + (i & ((1 << a.shift) - 1)); };
  if (keep >= L) {
    for (int i = tid; i < a.cap; i += SEL_THREADS) from[i] = -1;
    for (int i = tid; i < L; i += SEL_THREADS) {
      const size_t p = at(i);
      a.w_out[p] = a.w_in[p];
      a.b_out[p] = a.b_in[p];
    }
    return;
  }
  if (a.recent > 0) {
    int newest = INT_MIN;
    for (int i = tid; i < L; i += SEL_THREADS) newest = max(newest, a.b_in[at(i)]);
    newest = __reduce_max_sync(0xFFFFFFFFu, newest);
    if (lane == 0) atomicMax(&s_newest, newest);
    __syncthreads();
  }
  const long long after = (long long)s_newest - a.recent;  // positions above this are recent
  const bool held = L <= KEYS_SMEM;
  auto make_key = [&](int i) {
    const size_t p = at(i);
    if (a.recent > 0) {
      const long long age = (long long)a.b_in[p] - after;
      if (age > 0) return KEY_RECENT + (uint32_t)age;
    }
    return key_of(a.w_in[p]);
  };
  if (held) {
    for (int i = tid; i < L; i += SEL_THREADS) s_keys[i] = make_key(i);
  }
  auto key = [&](int i) { return held ? s_keys[i] : make_key(i); };
  // ---- the keep-th largest key
  uint32_t prefix = 0, mask = 0, want = (uint32_t)keep;  // keys of this prefix still wanted
#pragma unroll 1
  for (int pass = 0; pass < 3 && keep > 0; ++pass) {
    const int low = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
    for (int i = tid; i < BINS; i += SEL_THREADS) s_hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < L; i += SEL_THREADS) {
      const uint32_t k = key(i);
      if ((k & mask) == prefix) atomicAdd(&s_hist[(k >> low) & ((1u << bits) - 1u)], 1u);
    }
    __syncthreads();
    // the bin where the count from above reaches `want`: two bins a thread, from the top
    const uint32_t c0 = s_hist[BINS - 1 - 2 * tid], c1 = s_hist[BINS - 2 - 2 * tid];
    uint32_t inc = c0 + c1;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, inc, o);
      if (lane >= o) inc += v;
    }
    if (lane == 31) s_sum[warp] = inc;
    __syncthreads();
    uint32_t base = 0;
    for (int w = 0; w < warp; ++w) base += s_sum[w];
    const uint32_t above = base + inc - c0 - c1;
    if (above < want && want <= above + c0) s_digit = BINS - 1 - 2 * tid, s_left = want - above;
    else if (above + c0 < want && want <= above + c0 + c1) s_digit = BINS - 2 - 2 * tid, s_left = want - above - c0;
    __syncthreads();
    prefix |= s_digit << low;
    mask |= ((1u << bits) - 1u) << low;
    want = s_left;
    __syncthreads();
  }
  // prefix: the smallest key that stays; `want` of its ties do, the first ones
  const uint32_t edge = keep > 0 ? prefix : 0xFFFFFFFFu;
  const int seg = ((L + SEL_WARPS - 1) / SEL_WARPS + 31) & ~31, i0 = min(L, warp * seg), i1 = min(L, i0 + seg);
  const uint32_t below = (1u << lane) - 1u;
  int ties = 0;
  for (int i = i0; i < i1; i += 32) ties += __popc(__ballot_sync(0xFFFFFFFFu, i + lane < i1 && key(i + lane) == edge));
  if (lane == 0) s_warp[warp][0] = ties;
  __syncthreads();
  int ties0 = 0;
  for (int w = 0; w < warp; ++w) ties0 += s_warp[w][0];
  // which of 32 tokens from i on stay; t: ties met so far
  auto stay = [&](int i, int& t) {
    const uint32_t k = i + lane < i1 ? key(i + lane) : 0u;
    const bool tie = i + lane < i1 && k == edge;
    const uint32_t ts = __ballot_sync(0xFFFFFFFFu, tie);
    const bool s = keep > 0 && i + lane < i1 && (k > edge || (tie && t + __popc(ts & below) < (int)want));
    t += __popc(ts);
    return __ballot_sync(0xFFFFFFFFu, s);
  };
  auto lows = [&](int i) { return keep <= i ? 0u : keep - i >= 32 ? 0xFFFFFFFFu : (1u << (keep - i)) - 1u; };  // places below keep
  int holes = 0, sources = 0, t = ties0;
  for (int i = i0; i < i1; i += 32) {
    const uint32_t s = stay(i, t), lo = lows(i);
    holes += __popc(~s & lo);
    sources += __popc(s & ~lo);
  }
  if (lane == 0) s_warp[warp][1] = holes, s_warp[warp][2] = sources;
  __syncthreads();
  int hole0 = 0, source0 = 0;
  for (int w = 0; w < warp; ++w) hole0 += s_warp[w][1], source0 += s_warp[w][2];
  t = ties0;
  for (int i = i0; i < i1; i += 32) {  // the sources, in order
    const uint32_t s = stay(i, t) & ~lows(i);
    if ((s >> lane) & 1u) list[source0 + __popc(s & below)] = i + lane;
    source0 += __popc(s);
  }
  __syncthreads();
  t = ties0;
  for (int i = i0; i < min(i1, keep); i += 32) {
    const uint32_t gone = ~stay(i, t) & lows(i);
    if (i + lane < keep) {
      const bool hole = (gone >> lane) & 1u;
      const int src = hole ? list[hole0 + __popc(gone & below)] : -1;
      from[i + lane] = src;
      const size_t p = at(i + lane), q = hole ? at(src) : p;
      a.w_out[p] = a.w_in[q];
      a.b_out[p] = a.b_in[q];
    }
    hole0 += __popc(gone);
  }
  for (int i = keep + tid; i < a.cap; i += SEL_THREADS) from[i] = -1;
}

// last = 0: every block but the one that holds index keep; 1: that one.
__global__ void __launch_bounds__(MV_THREADS) k_move(EvictArgs a, int last, int blocks) {
  const int lane = threadIdx.x & 31, half = lane >> 4, l16 = lane & 15;
  const uint32_t group = 0xFFFFu << (lane & 16);
  const long long item = (long long)blockIdx.x * MV_WARPS + (threadIdx.x >> 5), units = (long long)a.batch * a.Hkv;
  if (item >= (last ? units : units * blocks)) return;
  const long long unit = last ? item : item / blocks;
  const int b = (int)(unit / a.Hkv), h = (int)(unit - (long long)b * a.Hkv);
  const int keep = a.keep[b], L = a.kv_len[b];
  int t = last ? keep >> 4 : (int)(item - unit * blocks);
  if (keep < 0 || keep >= L || keep > a.cap || t * KV8_BLOCK >= keep || (t == keep >> 4) != (last != 0)) return;
  const int base = t * KV8_BLOCK;
  const int32_t* from = a.from + (size_t)unit * a.cap;
  const int mine = l16 + base < keep ? from[base + l16] : -1;
  if (!__any_sync(0xFFFFFFFFu, mine >= 0)) return;
  const int32_t* tab = a.table + (size_t)b * a.max_pages;
  auto at = [&](int i) { return ((((size_t)tab[i >> a.shift]) * a.Hkv + h) << a.shift) + (i & ((1 << a.shift) - 1)); };
  const size_t to = at(base);
  uint8_t* codes = half ? a.vc : a.kc;
  float* scales = half ? a.vs : a.ks;
  const int live = min(KV8_BLOCK, L - base);
  uint2 w[KV8_BLOCK];
  const size_t row_at = mine >= 0 ? at(mine) : to + l16;  // lane l16: where row l16 comes from
  const float row_scale = scales[row_at >> 4];
#pragma unroll
  for (int j = 0; j < KV8_BLOCK; ++j) {
    const size_t r = __shfl_sync(0xFFFFFFFFu, (unsigned long long)row_at, j);
    w[j] = j < live ? reinterpret_cast<const uint2*>(codes + r * HD)[l16] : make_uint2(0, 0);
  }
  // the largest magnitude, by the bytes' order, times 2^-6 so that none overflows
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < KV8_BLOCK; ++j) {
    const uint32_t m = __vmaxu4(w[j].x & 0x7F7F7F7Fu, w[j].y & 0x7F7F7F7Fu);
    const uint32_t m2 = max(max(m & 255u, (m >> 8) & 255u), max((m >> 16) & 255u, m >> 24));
    const float s = __shfl_sync(group, row_scale, j, 16);
    top = fmaxf(top, e4m3x2_floats(m2).x * kv8_pow2(min(max(kv8_exp(s), KV8_MIN_EXP), KV8_MAX_EXP) - 6));
  }
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) top = fmaxf(top, __shfl_xor_sync(group, top, o));
  const bool nan = __any_sync(group, l16 < live && kv8_nan(row_scale));
  const int e = nan ? 0 : max(kv8_exp_for(top) + 6, KV8_MIN_EXP);
  __syncwarp();
#pragma unroll
  for (int j = 0; j < KV8_BLOCK; ++j) {
    const float s = __shfl_sync(group, row_scale, j, 16);
    if (j >= live) continue;
    const int d = nan ? 0 : kv8_exp(s) - e;
    if (d != 0) {
      w[j].x = kv8_rescale4(w[j].x, d);
      w[j].y = kv8_rescale4(w[j].y, d);
    }
    reinterpret_cast<uint2*>(codes + (to + j) * HD)[l16] = w[j];
  }
  if (l16 == 0) scales[to >> 4] = nan ? __uint_as_float(0x7FC00000u) : kv8_pow2(e);
}

}  // namespace

extern "C" size_t fc_kv8_evict_workspace(int batch, int Hkv, int cap) {
  if (batch < 1 || Hkv < 1 || cap < 0) return 0;
  return (size_t)batch * Hkv * std::max(cap, 1) * sizeof(int32_t);
}

extern "C" fc_status fc_kv8_evict(const fc_kv8_cache* cache, const int32_t* d_table, int max_pages, const int32_t* d_kv_len,
                                  const int32_t* d_keep, int batch, int recent, const float* d_weight_in,
                                  const int32_t* d_born_in, float* d_weight_out, int32_t* d_born_out, int32_t* d_from, int cap,
                                  void* d_ws, size_t ws_bytes, fc_stream stream) {
  FC_NVTX_RANGE();
  if (const fc_status st = fc_kv8_check(cache)) return st;
  const int shift = kv8_page_shift(cache->page_size);
  if (batch < 0 || max_pages < 1 || recent < 0 || cap < 0) return FC_ERR_INVALID_ARG;
  if (recent > MAX_RECENT || (long long)max_pages << shift > 0x7FFFFFFFll || (long long)batch * cache->Hkv > 1 << 24)
    return FC_ERR_UNSUPPORTED;
  if (batch == 0) return FC_OK;
  if (!d_table || !d_kv_len || !d_keep || !d_weight_in || !d_born_in || !d_weight_out || !d_born_out || (cap && !d_from) ||
      d_weight_in == d_weight_out || d_born_in == d_born_out)
    return FC_ERR_INVALID_ARG;
  if (!d_ws || !kv8_aligned(d_ws, 4) || ws_bytes < fc_kv8_evict_workspace(batch, cache->Hkv, cap)) return FC_ERR_WORKSPACE;
  EvictArgs a{d_table, d_kv_len, d_keep, max_pages, cache->n_pages, shift, cache->Hkv, batch, cap, recent, d_weight_in, d_born_in,
              d_weight_out, d_born_out, d_from, static_cast<int32_t*>(d_ws), static_cast<uint8_t*>(cache->k_codes),
              static_cast<uint8_t*>(cache->v_codes), static_cast<float*>(cache->k_scale), static_cast<float*>(cache->v_scale),
              fc_error_slot()};
  static std::atomic<unsigned long long> done{0};
  const fc_status st = fc_once_per_device(done, [](int) {
    return fc_cuda_status(cudaFuncSetAttribute(k_select, cudaFuncAttributeMaxDynamicSharedMemorySize, KEYS_SMEM * 4));
  });
  if (st != FC_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const long long units = (long long)batch * cache->Hkv, longest = (long long)max_pages << shift;
  k_select<<<(unsigned)units, SEL_THREADS, (size_t)std::min<long long>(longest, KEYS_SMEM) * 4, s>>>(a);
  if (cap > 0) {
    const int blocks = (cap + KV8_BLOCK - 1) / KV8_BLOCK;
    const long long warps = units * blocks;
    if ((warps + MV_WARPS - 1) / MV_WARPS > 0x7FFFFFFFll) return FC_ERR_UNSUPPORTED;
    k_move<<<(unsigned)((warps + MV_WARPS - 1) / MV_WARPS), MV_THREADS, 0, s>>>(a, 0, blocks);
    k_move<<<(unsigned)((units + MV_WARPS - 1) / MV_WARPS), MV_THREADS, 0, s>>>(a, 1, blocks);
  }
  return FC_CHECK_LAUNCH();
}
