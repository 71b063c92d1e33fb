// Keys and values rounded into the pages of the 8-bit cache and read back
// (fc_kv8_write, fc_kv8_read).
#include <algorithm>

#include "kv8.cuh"

FC_DEFINE_ERROR_WORD(kv8)

namespace {

constexpr int HD = KV8_D;
constexpr int WR_THREADS = 256, WR_WARPS = WR_THREADS / 32;
constexpr int WINDOW = 32;  // rows of a block lie within so many rows of one another
constexpr long long MAX_ITEMS = 1ll << 30;

struct Kv8Rows {
  const __nv_bfloat16 *k, *v;
  int n_per_seq, n_src;
  bool one_seq;
  int64_t seq_stride, row_stride, head_stride;
};

struct Kv8Write {
  Kv8Rows x;
  const int32_t *src, *slot, *pos;
  int rows, Hkv, shift;
  long long n_slots;
  uint8_t *kc, *vc;
  float *ks, *vs;
  float* weight;
  int32_t* born;
  unsigned int* err;
};

// A warp takes `per` neighbouring rows of one head, keys or values.  A row begins a run when
// none of the WINDOW rows before it goes to its block of 16; the run's rows are it and
// those of the next WINDOW that do.  So the warp that meets a run's first row
// knows the whole block's new tokens, and no two warps write one block.
// Four dimensions a lane, the block's 16 places at once: their largest magnitude (bf16 bits as unsigned numbers order
// like the magnitudes, infinities and NaN on top) gives the scale.  Lane j works
// out where place j's row is, for all (59400 x 8 rows 68 us, 5.4 TB/s; with every
// lane working out every place's 89, and 176 before places were looked up by
// their rows).  What a block holds in flight bounds it, 16 rows a warp at 62
// registers, next to its instructions (68% of the issue slots).
__global__ void __launch_bounds__(WR_THREADS) k_kv8_write(Kv8Write a, int per) {
  __shared__ int s_row[WR_WARPS][KV8_BLOCK];
  const int lane = threadIdx.x & 31;
  const bool values = threadIdx.x & 32;
  const long long item = (long long)blockIdx.x * (WR_WARPS / 2) + (threadIdx.x >> 6);
  const int h = (int)(item % a.Hkv);
  const long long r0l = item / a.Hkv * per;
  if (r0l >= a.rows) return;
  const int r0 = (int)r0l;
  // the place that a row goes to, -1: none
  auto place = [&](int r) {
    if (r < 0 || r >= a.rows) return -1;
    const int sl = a.slot[r];
    if (sl < 0) return -1;
    const int at = a.src ? a.src[r] : r;
    return sl < a.n_slots && at >= 0 && at < a.x.n_src ? sl : -1;
  };
  int* row_of = s_row[threadIdx.x >> 5];
  const __nv_bfloat16* x0 = (values ? a.x.v : a.x.k) + h * a.x.head_stride;
  uint8_t* codes = values ? a.vc : a.kc;
  float* scales = values ? a.vs : a.ks;
  const int before = place(r0 - WINDOW + lane), here = place(r0 + lane), next = place(r0 + WINDOW + lane);
  if (h == 0 && !values && lane < per && r0 + lane < a.rows && here < 0 && a.slot[r0 + lane] >= 0) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_INVALID);
  const int last = __shfl_sync(0xFFFFFFFFu, before, 31), up = __shfl_up_sync(0xFFFFFFFFu, here, 1);
  // rows whose neighbour above goes elsewhere
  uint32_t starts = __ballot_sync(0xFFFFFFFFu, lane < per && here >= 0 && here >> 4 != (lane ? up : last) >> 4);
#pragma unroll 1
  for (; starts; starts &= starts - 1) {
    const int i = __ffs(starts) - 1, mine = __shfl_sync(0xFFFFFFFFu, here, i), block = mine >> 4;
    // rows r0 + i - WINDOW .. - 1, then r0 + i .. + WINDOW
    const uint32_t same_b = __ballot_sync(0xFFFFFFFFu, before >> 4 == block);
    const uint32_t same_h = __ballot_sync(0xFFFFFFFFu, here >> 4 == block);
    if ((same_b >> i) | (same_h & ((1u << i) - 1u))) continue;  // an earlier row's run
    if (lane < KV8_BLOCK) row_of[lane] = -1;
    __syncwarp();
    if (lane >= i && here >> 4 == block) row_of[here & 15] = r0 + lane;
    if (lane <= i && next >> 4 == block) row_of[next & 15] = r0 + WINDOW + lane;
    __syncwarp();
    const int page = mine >> a.shift, in_page = (mine & ((1 << a.shift) - 1)) >> 4;
    const size_t row0 = (((size_t)page * a.Hkv + h) << a.shift) + in_page * KV8_BLOCK;
    const int my_row = lane < KV8_BLOCK ? row_of[lane] : -1;
    const uint32_t have = __ballot_sync(0xFFFFFFFFu, my_row >= 0);  // places that get a row
    const int first = __ffs(have) - 1;
    long long from = 0;
    if (my_row >= 0) {
      const int at = a.src ? a.src[my_row] : my_row, q = a.x.one_seq ? 0 : at / a.x.n_per_seq, n = at - q * a.x.n_per_seq;
      from = q * a.x.seq_stride + n * a.x.row_stride;
      if (a.weight && !values) {
        a.weight[row0 + lane] = 0.f;
        a.born[row0 + lane] = a.pos[my_row];
      }
    }
    float* scale = scales + (row0 >> 4);
    uint32_t* rows = reinterpret_cast<uint32_t*>(codes + row0 * HD) + lane;
    uint2 v[KV8_BLOCK];
#pragma unroll
    for (int j = 0; j < KV8_BLOCK; ++j) {
      const long long off = __shfl_sync(0xFFFFFFFFu, from, j);
      v[j] = make_uint2(0, 0);
      if ((have >> j) & 1u) v[j] = __ldcs(reinterpret_cast<const uint2*>(x0 + off) + lane);
    }
    const float old = first > 0 ? *scale : 0.f;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < KV8_BLOCK; ++j) top = __vmaxu2(top, __vmaxu2(v[j].x & 0x7FFF7FFFu, v[j].y & 0x7FFF7FFFu));
    top = __reduce_max_sync(0xFFFFFFFFu, max(top & 0xFFFFu, top >> 16));
    const bool nan = top >= 0x7F80u || kv8_nan(old);
    int e = nan ? 0 : max(kv8_exp_for(__uint_as_float(top << 16)), KV8_MIN_EXP);
    if (first > 0 && !nan) {
      const int e_old = kv8_exp(old);
      if (e > e_old) {  // what the block holds, in the new scale
#pragma unroll 4
        for (int j = 0; j < first; ++j) rows[j * 32] = kv8_times4(rows[j * 32], kv8_half_pow2(e_old - e));
      } else {
        e = e_old;
      }
    }
    __syncwarp();  // all have read the scale
    if (lane == 0) *scale = nan ? __uint_as_float(0x7FC00000u) : kv8_pow2(e);
    const float by = kv8_pow2(-e);
#pragma unroll
    for (int j = 0; j < KV8_BLOCK; ++j) {
      auto two = [&](uint32_t w) { return floats_e4m3x2(__uint_as_float(w << 16) * by, __uint_as_float(w & 0xFFFF0000u) * by); };
      // a block with a NaN or an infinity stands for NaN, whatever its numbers
      if ((have >> j) & 1u) rows[j * 32] = nan ? 0u : two(v[j].x) | (two(v[j].y) << 16);
    }
    __syncwarp();  // the places' rows are read before the next run's
  }
}

// A row and head 16 lanes, 16 bytes in and 32 out each: 59400 x 8 rows 63 us, 5.8 TB/s.
__global__ void __launch_bounds__(WR_THREADS) k_kv8_read(const int32_t* __restrict__ slot, int rows, int Hkv, int shift, long long n_slots,
                                                         const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
                                                         const float* __restrict__ ks, const float* __restrict__ vs, uint4* __restrict__ k,
                                                         uint4* __restrict__ v, unsigned int* err) {
  const int lane = threadIdx.x & 15;  // 16 lanes a (row, head)
  const long long items = (long long)rows * Hkv, stride = (long long)gridDim.x * (WR_THREADS / 16);
  for (long long it = (long long)blockIdx.x * (WR_THREADS / 16) + threadIdx.x / 16; it < items; it += stride) {
    const int r = (int)(it / Hkv), h = (int)(it - (long long)r * Hkv);
    const int sl = slot[r];
    if (sl >= n_slots && lane == 0 && h == 0) fc_flag(FC_ERR_WORD(err), FC_EBIT_INVALID);
    uint2 a = make_uint2(0, 0), b = a;
    float sk = 0.f, sv = 0.f;
    if (sl >= 0 && sl < n_slots) {
      const size_t row = ((((size_t)(sl >> shift)) * Hkv + h) << shift) + (sl & ((1 << shift) - 1));
      a = reinterpret_cast<const uint2*>(kc)[row * 16 + lane];
      b = reinterpret_cast<const uint2*>(vc)[row * 16 + lane];
      sk = ks[row >> 4];
      sv = vs[row >> 4];
    }
    auto values = [](const uint2& w, float s) {  // four significant bits times a power of two: exact in bf16's range
      const float2 p = e4m3x2_floats(w.x & 0xFFFFu), q = e4m3x2_floats(w.x >> 16), t = e4m3x2_floats(w.y & 0xFFFFu), u = e4m3x2_floats(w.y >> 16);
      return make_uint4(pack_bf16x2(p.x * s, p.y * s), pack_bf16x2(q.x * s, q.y * s), pack_bf16x2(t.x * s, t.y * s), pack_bf16x2(u.x * s, u.y * s));
    };
    const size_t to = (size_t)it * 16 + lane;
    __stcs(k + to, values(a, sk));
    __stcs(v + to, values(b, sv));
  }
}

}  // namespace

fc_status fc_kv8_check(const fc_kv8_cache* c) {
  if (!c || c->n_pages < 1 || c->Hkv < 1) return FC_ERR_INVALID_ARG;
  if (c->D != HD || kv8_page_shift(c->page_size) < 0 || (long long)c->n_pages * c->page_size > 0x7FFFFFFFll ||
      (long long)c->n_pages * c->page_size * c->Hkv > 0x7FFFFFFFll)  // rows are counted in 32 bits (256 GB of codes)
    return FC_ERR_UNSUPPORTED;
  if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !kv8_aligned(c->k_codes, 32) || !kv8_aligned(c->v_codes, 32) ||
      !kv8_aligned(c->k_scale, 4) || !kv8_aligned(c->v_scale, 4))
    return FC_ERR_INVALID_ARG;
  return FC_OK;
}

extern "C" fc_status fc_kv8_write(const fc_kv8_cache* cache, const void* d_k, const void* d_v, int n_seq, int n_per_seq,
                                  int64_t seq_stride, int64_t row_stride, int64_t head_stride, const int32_t* d_src,
                                  const int32_t* d_slot, int rows, const int32_t* d_pos, float* d_weight, int32_t* d_born,
                                  fc_stream stream) {
  FC_NVTX_RANGE();
  if (const fc_status st = fc_kv8_check(cache)) return st;
  if (rows < 0 || n_seq < 0 || n_per_seq < 1 || seq_stride < 0 || row_stride < 0 || head_stride < 0 ||
      (long long)n_seq * n_per_seq > 0x7FFFFFFFll || !d_weight != !d_born || (d_weight && !d_pos && rows))
    return FC_ERR_INVALID_ARG;
  if (rows == 0) return FC_OK;
  if (!d_k || !d_v || !d_slot || !kv8_aligned(d_k, 16) || !kv8_aligned(d_v, 16) || seq_stride % 8 || row_stride % 8 ||
      head_stride % 8 || (!d_src && rows > n_seq * n_per_seq))
    return FC_ERR_INVALID_ARG;
  if ((long long)rows * cache->Hkv > MAX_ITEMS) return FC_ERR_UNSUPPORTED;
  Kv8Write a{{static_cast<const __nv_bfloat16*>(d_k), static_cast<const __nv_bfloat16*>(d_v), n_per_seq, n_seq * n_per_seq,
              n_seq == 1, seq_stride, row_stride, head_stride},
             d_src, d_slot, d_pos, rows, cache->Hkv, kv8_page_shift(cache->page_size),
             (long long)cache->n_pages * cache->page_size, static_cast<uint8_t*>(cache->k_codes),
             static_cast<uint8_t*>(cache->v_codes), static_cast<float*>(cache->k_scale), static_cast<float*>(cache->v_scale),
             d_weight, d_born, fc_error_slot()};
  // one row a warp while that does not fill the GPU, else a block's worth
  const int per = (long long)rows * cache->Hkv <= 152 * 64 ? 1 : 16;
  const long long warps = ((long long)rows + per - 1) / per * cache->Hkv;
  k_kv8_write<<<(unsigned)((2 * warps + WR_WARPS - 1) / WR_WARPS), WR_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(a, per);
  return FC_CHECK_LAUNCH();
}

extern "C" fc_status fc_kv8_read(const fc_kv8_cache* cache, const int32_t* d_slot, int rows, void* d_k, void* d_v,
                                 fc_stream stream) {
  FC_NVTX_RANGE();
  if (const fc_status st = fc_kv8_check(cache)) return st;
  if (rows < 0) return FC_ERR_INVALID_ARG;
  if (rows == 0) return FC_OK;
  if (!d_slot || !d_k || !d_v || !kv8_aligned(d_k, 16) || !kv8_aligned(d_v, 16)) return FC_ERR_INVALID_ARG;
  const long long items = (long long)rows * cache->Hkv;
  if (items > MAX_ITEMS) return FC_ERR_UNSUPPORTED;
  const unsigned grid = (unsigned)std::min<long long>((items + WR_THREADS / 16 - 1) / (WR_THREADS / 16), 152 * 64);
  k_kv8_read<<<grid, WR_THREADS, 0, static_cast<cudaStream_t>(stream)>>>(
      d_slot, rows, cache->Hkv, kv8_page_shift(cache->page_size), (long long)cache->n_pages * cache->page_size,
      static_cast<const uint8_t*>(cache->k_codes), static_cast<const uint8_t*>(cache->v_codes),
      static_cast<const float*>(cache->k_scale), static_cast<const float*>(cache->v_scale), static_cast<uint4*>(d_k),
      static_cast<uint4*>(d_v), fc_error_slot());
  return FC_CHECK_LAUNCH();
}
