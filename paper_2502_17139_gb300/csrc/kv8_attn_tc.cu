// fc_kv8_attn for more than 16 query rows a kv head (draft trees, chunks): the
// tensor cores' products over the paged 8-bit cache.
//
// A unit is up to 256 query rows of one (sequence, kv head) and all its keys,
// in blocks of 128 keys, the new tokens the last.  Per block
//   S = Q K^T,  P = 2^(c S - m),  O += P V.
// The first product is in e4m3, the cache's rows as they are: TMA brings them
// from the pages into the operand's place, and no thread touches a key.  A query
// row, bf16 times a power of two, is the sum of two e4m3 rows: the nearest e4m3
// number leaves a remainder of at most four significant bits.  Two products at
// twice bf16's rate take bf16's time, and are exact for values down to 2^-9 of
// the row's largest.  New keys are split likewise.  A block's scale, 16 keys',
// multiplies scores.  The second product is in bf16, P needing its range: V's
// numbers times their scale, exact, as scales are powers of two.
//   * One warp looks the pages up, keeps the scales and asks for the keys' rows
//     (TMA) and, into L2, the values', up to four blocks ahead.
//   * Eight warps turn values into bf16 tiles in shared memory (128-byte
//     swizzle), two stages, one block ahead in registers: a byte's low seven
//     bits in bits 4..10 of a half are its magnitude times 2^-120 in bf16, and
//     one packed product with 2^120 times the scale, exact, makes it the value.
//   * One warp issues every tcgen05.mma (accumulators and P in tensor memory).
//   * Two softmax warpgroups, a row a thread.  With more than 128 rows each has
//     its tile and both take every block; with fewer both have the same rows,
//     one takes the even blocks and one the odd, and their halves are joined
//     at the end, so that one tile's softmax always has the other's products
//     beside it.
//   * The eight warps also fetch a unit's queries, while the last one's end is
//     written.
// The CTAs (one an SM) share all units' blocks equally, cut anywhere; a cut
// unit's pieces go through the workspace to k_kv8_join.
// Several roles run at once from one instruction cache, so the loops are short.
// Measured: 32 trees of 128 nodes, 4 query heads a kv head, over 16384 keys 899 us (1223
// TFLOP/s), 16 ragged trees of 64 nodes, a kv head a query head, 118 us.  What bounds it is a
// block's chain: of 4.0 K cycles a block of two tiles, a tile's weights take 2.3 K (a warp's instructions one
// after another, not a pipe), its products 1.0 K, hand-overs the rest; the tiles run side by side.
// Every mbarrier wait is bounded: one that runs out raises FC_ERR_TIMEOUT, the
// CTA lets its issued products and copies finish, frees its tensor memory and returns.
#include <algorithm>
#include <atomic>
#include <mutex>

#include "fc_common.cuh"
#include "kv8_attn.cuh"

FC_DEFINE_ERROR_WORD(kv8_tc)

namespace {

constexpr int HD = KV8_D;
constexpr int THREADS = 640;  // warp 0 products, 1 pieces, 2 scales and keys, 4-7 / 8-11 softmax, 12-19 queries and values to tiles
constexpr int NUM_WARPS = 8;
constexpr int QN = 2;  // queries' rows in hand a lane
constexpr int BM = 128, BN = 128, ROWS = 2 * BM;
constexpr uint32_t HALF_BYTES = 128 * 128;             // 64 bf16 dims, or all 128 e4m3 ones, of 128 rows
constexpr uint32_t TILE_BYTES = 2 * HALF_BYTES;        // a bf16 tile, or an e4m3 one's two parts
constexpr int SLOTS = 4;                               // blocks whose keys, scales and keep bits are kept
constexpr uint32_t OFF_Q = 0;                          // two tiles of two parts
constexpr uint32_t OFF_K = OFF_Q + 2 * TILE_BYTES;     // [SLOTS] keys
constexpr uint32_t OFF_K2 = OFF_K + SLOTS * HALF_BYTES;  // the new keys' second part
constexpr uint32_t OFF_V = OFF_K2 + HALF_BYTES;        // two stages
constexpr uint32_t OFF_KEEP = OFF_V + 2 * TILE_BYTES;  // [slot][4] bits of the keys that count
constexpr uint32_t OFF_BACK = OFF_KEEP + SLOTS * 16;   // [slot][8] what 16 keys' scores are to be multiplied by
constexpr uint32_t OFF_RUN = OFF_BACK + SLOTS * 32;    // [slot][8] where 16 keys' rows are, in runs of 16 rows
constexpr uint32_t OFF_VS = OFF_RUN + SLOTS * 32;      // [slot][8] 16 values' scale
constexpr int PIECES = 4;                              // piece descriptions kept
constexpr uint32_t OFF_QE = OFF_VS + SLOTS * 32;       // [PIECES][256] what a query row's scores are to be multiplied by
constexpr uint32_t OFF_ML = OFF_QE + PIECES * ROWS * 4;  // [2 turns][2][128] (m, l) exchanged at a unit's end
constexpr uint32_t OFF_BAD = OFF_ML + 4 * BM * 8;      // [PIECES][8] bits of the new tokens whose values are not finite
constexpr uint32_t OFF_PIECE = OFF_BAD + PIECES * 16;  // [PIECES]
constexpr uint32_t OFF_BAR = OFF_PIECE + PIECES * 64;
constexpr uint32_t SMEM_BYTES = OFF_BAR + 512 + 1024;  // + alignment slack
static_assert(SMEM_BYTES <= 232448, "shared memory");
constexpr uint32_t TMEM_COLS = 512;                             // S_0, S_1, O_0, O_1
constexpr uint64_t WAIT_CYCLES = 4000000000ull;                 // ~2 s
constexpr uint64_t DRAIN_CYCLES = 400000000ull;
constexpr float RESCALE_THRESHOLD = 8.f;  // O is rescaled when a row's maximum (base 2) grows by more
constexpr int E_TOP = 7;  // a query row's largest value, 16 new keys' largest, is put at 2^7..2^8
constexpr float M_START = -1e30f;  // a reference before any key
// Exponents of queries and new keys are taken as they are where 2^(e - E_TOP) and
// its inverse are normal fp32 numbers; smaller ones count as E_MIN (what a row of
// queries below it loses, 2^-136 a value, moves a score by less than 2^-23 beside
// keys of 448 * 2^100).  What a score is multiplied by, the row's factor times
// the keys', may underflow: it is at least FACTOR_MIN, and the row's at least
// ROW_MIN, as a factor of 0 would make NaN of masked scores, -infinity (sums of
// products are below 2^26, so that such a score is 0 beside 1).  And it is finite, as
// a sum of 0 between large queries and large keys is a score of 0.
constexpr int E_MIN = -119, E_MAX = 127;
constexpr float FACTOR_MIN = 0x1p-126f, ROW_MIN = 0x1p-149f, FACTOR_MAX = 0x1.fffffep127f;
// A unit's start and end in blocks of one tile: 4 where a unit is cut over CTAs (3
// requests of 128 nodes, 32 heads of their own, over 3000 keys 44 us, with 8 47), 7
// where a CTA has several (16 ragged trees of 64 nodes 117 us, with 12 123).  And
// the least share worth a CTA (32 nodes over 2000 keys 22.7 us, with 6 24).
constexpr int CUT_COST = 4, WHOLE_COST = 7, LEAST = 4;

// Registers a thread by warpgroup (setmaxnreg), of the launch's 96.  The shares must add up to the launch's
// allocation, or the increase never returns; the host checks the compiled count.
constexpr int REGS_LAUNCH = 96, REGS_ISSUE = 80, REGS_NUMBERS = 80, REGS_SOFTMAX = 120;
static_assert(REGS_ISSUE + 2 * REGS_NUMBERS + 2 * REGS_SOFTMAX <= 5 * REGS_LAUNCH, "register split");

enum {
  B_KFULL = 0,   // [SLOTS] 8 arrivals and their bytes, or 8 warps' of the new tokens
  B_VFULL = 4,   // [2] 8
  B_VEMPTY = 6,  // [2]
  B_SFULL = 8,   // [2 tiles]
  B_PFULL = 10,  // [2 tiles] 4
  B_INFO = 12,   // [SLOTS] a block's scales and keep bits
  B_SLOT = 16,   // [SLOTS] a slot's block is done with
  B_PIECE = 20,  // [PIECES] a description is written
  B_QFULL = 24,  // [PIECES] 9
  B_QE = 28,     // [PIECES] 8: the query rows' factors
  B_QFREE = 32,
  B_OFIN = 33,
  B_OFREE = 34,  // 256
  B_ML = 35,     // 256: a row's halves exchanged
  B_DRAIN = 36,
  N_BARS = 37
};

struct ManyArgs {
  Kv8Args a;
  int chunks;      // most units a (sequence, kv head)
  int split;       // 0: whole units, CTA by CTA
  int unit_cost;   // CUT_COST or WHOLE_COST
  int rows_cap;    // rows a piece's slot has room for
  uint32_t by_G;   // r / G is r * by_G >> 20 for r < 2048
  int* list;       // [grid][8] cut units for k_kv8_join
  float* part_o;   // [grid][2][rows_cap][HD]
  float2* part_ml; // [grid][2][rows_cap]
  __device__ __forceinline__ int node_of(int r) const { return (int)((uint32_t)r * by_G >> 20); }
};

__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort) {
  return __all_sync(0xFFFFFFFFu, mbar_wait_bounded(bar, parity, abort, WAIT_CYCLES));
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint64_t f2_pack(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void f2_unpack(uint64_t v, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float max_nan(float a, float b) {  // NaN of either
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float d;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// 16 rows of 32 columns: register 4i + 2k + e is column 8i + 2 (lane % 4) + e of row lane / 4 + 8k
__device__ __forceinline__ void tmem_ld_rows(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
template <int N>
__device__ __forceinline__ void regs_dec() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_inc() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
// The products of a tile and a block, one lane elected for all of a statement's:
// descriptors differ in their low words, by constants; their high words are
// alike (1024 bytes between 8-row groups, version 1, 128-byte swizzle).  One
// statement, so that the operands move to uniform registers once.
constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
// S[tmem d] (+)= A . B^T, e4m3 tiles in shared memory, 128 dims K-major: four of K = 32
__device__ __forceinline__ void mma_qk(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred z, o, e;\n\t.reg .b64 a, b;\n\t.reg .b32 t, h;\n\tmov.b32 h, %5;\n\t"
      "setp.ne.b32 z, %4, 0;\n\tsetp.eq.b32 o, 0, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
      "add.u32 t, %1, 0;\n\tmov.b64 a, {t, h};\n\tadd.u32 t, %2, 0;\n\tmov.b64 b, {t, h};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %3, z;\n\t"
      "add.u32 t, %1, 2;\n\tmov.b64 a, {t, h};\n\tadd.u32 t, %2, 2;\n\tmov.b64 b, {t, h};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %3, o;\n\t"
      "add.u32 t, %1, 4;\n\tmov.b64 a, {t, h};\n\tadd.u32 t, %2, 4;\n\tmov.b64 b, {t, h};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %3, o;\n\t"
      "add.u32 t, %1, 6;\n\tmov.b64 a, {t, h};\n\tadd.u32 t, %2, 6;\n\tmov.b64 b, {t, h};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %3, o;\n\t"
      "}" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(add), "n"(DESC_HI)
      : "memory");
}
// O[tmem d] (+)= P[tmem a] . V, V's rows (keys) in shared memory
__device__ __forceinline__ void mma_pv(uint32_t d, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred z, o, e;\n\t.reg .b64 b;\n\t.reg .b32 t, h;\n\tmov.b32 h, %5;\n\t"
      "setp.ne.b32 z, %4, 0;\n\tsetp.eq.b32 o, 0, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
      "add.u32 t, %2, 0;\n\tmov.b64 b, {t, h};\n\tadd.u32 t, %1, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [t], b, %3, z;\n\t"
      "add.u32 t, %2, 128;\n\tmov.b64 b, {t, h};\n\tadd.u32 t, %1, 8;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [t], b, %3, o;\n\t"
      "add.u32 t, %2, 256;\n\tmov.b64 b, {t, h};\n\tadd.u32 t, %1, 16;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [t], b, %3, o;\n\t"
      "add.u32 t, %2, 384;\n\tmov.b64 b, {t, h};\n\tadd.u32 t, %1, 24;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [t], b, %3, o;\n\t"
      "add.u32 t, %2, 512;\n\tmov.b64 b, {t, h};\n\tadd.u32 t, %1, 32;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [t], b, %3, o;\n\t"
      "add.u32 t, %2, 640;\n\tmov.b64 b, {t, h};\n\tadd.u32 t, %1, 40;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [t], b, %3, o;\n\t"
      "add.u32 t, %2, 768;\n\tmov.b64 b, {t, h};\n\tadd.u32 t, %1, 48;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [t], b, %3, o;\n\t"
      "add.u32 t, %2, 896;\n\tmov.b64 b, {t, h};\n\tadd.u32 t, %1, 56;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [t], b, %3, o;\n\t"
      "}" ::"r"(d),
      "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(add), "n"(DESC_HI)
      : "memory");
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;\n" ::: "memory"); }
// 32 bytes at once (by 16 each sector is asked for twice: 16 ragged trees of 64 nodes 121 us instead of 117)
__device__ __forceinline__ void ld_global32(uint4& a, uint4& b, const void* p) {
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w)
               : "l"(p));
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
// Largest finite magnitude of a word's two bf16 values, packed like them.
__device__ __forceinline__ uint32_t top2(uint32_t top, uint32_t w) {
  const uint32_t mag = w & 0x7FFF7FFFu;
  return __vmaxu2(top, mag & ~__vcmpgeu2(mag, 0x7F807F80u));
}
// Exponent of a magnitude given as bf16 bits, in E_MIN..E_MAX.
__device__ __forceinline__ int expo_of(uint32_t bits) { return min(max((int)(bits >> 7) - 127, E_MIN), E_MAX); }
// 8 bf16 values times a power of two as the sum of two e4m3 rows' bytes.  The
// nearest e4m3 number has four significant bits, so it leaves at most four of
// the eight, in steps that e4m3 has down to 2^-9.
__device__ __forceinline__ void split8(const uint4& v, float by, uint2& p1, uint2& p2) {
  uint32_t a[4], b[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const uint32_t w = (&v.x)[u];
    float x = lo_f(w) * by, y = hi_f(w) * by;
    x = fmaf(x, 0.f, x), y = fmaf(y, 0.f, y);  // an infinity becomes NaN, not 448
    a[u] = floats_e4m3x2(x, y);
    const float2 near = e4m3x2_floats(a[u]);
    b[u] = floats_e4m3x2(x - near.x, y - near.y);
  }
  p1 = make_uint2(a[0] | (a[1] << 16), a[2] | (a[3] << 16));
  p2 = make_uint2(b[0] | (b[1] << 16), b[2] | (b[3] << 16));
}

// The first (sel 0x1000) or last two (0x3020) cached numbers of each word, times 2^-120 times f1 (times f2), as bf16
__device__ __forceinline__ uint4 values8(uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t sel, uint32_t f1, uint32_t f2) {
  auto two = [&](uint32_t w) {
    const uint32_t x = __byte_perm(w, w, sel);
    uint32_t r = ((x >> 4) & 0x07F007F0u) | (x & 0x80008000u);
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(r), "r"(f1));
    if (f2 != 0x3F803F80u) asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(r), "r"(f2));
    return r;
  };
  return make_uint4(two(a), two(b), two(c), two(d));
}

// A CTA's part of a unit: n blocks from s0 on (n = 0: there is no more).
struct Piece {
  int b, gh, row0, rows, nn, kvl, cached, s0, n;
  int two;    // the softmax warpgroups have different rows
  int whole;  // all of the unit's blocks
  int slot;   // else where its sums go
};
static_assert(sizeof(Piece) <= 64, "piece description");

// Where a piece's queries are: a piece of one tile that follows another takes
// the other of the two tiles, so that its queries need not wait for the last
// piece's products (those of the piece before it are complete, else it would
// not have been described).
struct QTile {
  int tile = 0;
  bool alone = false;  // the last piece had one tile
  // true: the last piece's products must be complete first
  __device__ __forceinline__ bool next(bool two) {
    const bool other = alone && !two;
    tile = other ? 1 - tile : 0;
    alone = !two;
    return !other;
  }
};

// The units' blocks dealt out.  One warp of a CTA walks them and leaves each
// piece's description in shared memory for the other roles.
struct Walk {
  const ManyArgs& f;
  KvCut cut;
  int cur, end, b, base;  // balanced: position, end, request, its first cost; whole units: unit, units
  // the piece: blocks [s0, s1) of the unit's `blocks`
  int gh, chunk, nn, kvl, R, row0, rows, cached, blocks, s0, s1, unit_base, cost;
  bool bad, two;  // two: both softmax warpgroups' rows differ

  struct Req {
    int nn, kvl, R, n_chunks, rows_each, cached, blocks, w;
    bool bad;
  };
  // chunk sizes are equal, so that a request's units cost the same
  __device__ __forceinline__ Req req(int i) const {
    const Kv8Args& a = f.a;
    Req r;
    r.kvl = a.kv_len[i];
    r.nn = a.n_nodes ? a.n_nodes[i] : a.n_pad;
    r.bad = r.nn < 0 || r.nn > a.n_pad || r.kvl < 0 || r.kvl > (long long)a.max_pages << a.shift;
    if (r.bad) r.nn = r.kvl = 0;
    r.R = r.nn * a.G;
    r.n_chunks = max(1, (r.R + ROWS - 1) / ROWS);
    r.rows_each = (r.R + r.n_chunks - 1) / r.n_chunks;
    r.cached = r.R ? (int)(((uint32_t)r.kvl + BN - 1) / BN) : 0;  // lengths up to 2^31 - 1
    r.blocks = max(1, r.cached + (a.k_new && r.R ? 1 : 0));
    r.w = r.rows_each > BM ? 2 : 1;
    return r;
  }
  __device__ __forceinline__ int unit_cost(const Req& r) const { return f.unit_cost + r.blocks * r.w; }

  // every lane of a warp calls this
  __device__ __forceinline__ Walk(const ManyArgs& args) : f(args), cut(1, 1, 1) {
    const Kv8Args& a = f.a;
    const int lane = threadIdx.x & 31;
    b = 0;
    base = 0;
    if (!f.split) {
      cur = blockIdx.x;
      end = a.B * a.Hkv * f.chunks;
      return;
    }
    auto cost_of = [&](int i) {
      const Req r = req(i);
      return unit_cost(r) * r.n_chunks * a.Hkv;
    };
    const int first = lane < a.B ? cost_of(lane) : 0;
    int sum = first;
#pragma unroll 1
    for (int i = lane + 32; i < a.B; i += 32) sum += cost_of(i);
    cut = KvCut(__reduce_add_sync(0xFFFFFFFFu, sum), gridDim.x, LEAST);
    cur = (int)blockIdx.x < cut.n ? cut.start(blockIdx.x) : 0;
    end = (int)blockIdx.x < cut.n ? cut.start(blockIdx.x + 1) : 0;
#pragma unroll 1
    for (int b0 = 0; b0 < a.B; b0 += 32) {
      const int mine = b0 == 0 ? first : (b0 + lane < a.B ? cost_of(b0 + lane) : 0);
      int inc = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, inc, o);
        if (lane >= o) inc += v;
      }
      const uint32_t hit = __ballot_sync(0xFFFFFFFFu, base + inc > cur);
      if (hit) {
        const int w = __ffs(hit) - 1;
        b = b0 + w;
        base += __shfl_sync(0xFFFFFFFFu, inc - mine, w);
        break;
      }
      base += __shfl_sync(0xFFFFFFFFu, inc, 31);
    }
  }

  // the next piece of this CTA; false when there is none
  __device__ __forceinline__ bool next() {
    const Kv8Args& a = f.a;
    for (;;) {
      if (cur >= end) return false;
      Req r;
      if (f.split) {
        r = req(b);
        while (cur - base >= unit_cost(r) * r.n_chunks * a.Hkv) {
          base += unit_cost(r) * r.n_chunks * a.Hkv;
          ++b;
          r = req(b);
        }
        cost = unit_cost(r);
        const int u = (cur - base) / cost;
        gh = u / r.n_chunks;
        chunk = u - gh * r.n_chunks;
        unit_base = base + u * cost;
        // a block belongs to the share that holds its first cost
        const int from = max(0, cur - unit_base - f.unit_cost), to = min(cost, end - unit_base) - f.unit_cost;
        s0 = (from + r.w - 1) / r.w;
        s1 = to <= 0 ? 0 : (to + r.w - 1) / r.w;
        cur = min(unit_base + cost, end);
      } else {
        const int u = cur;
        cur += gridDim.x;
        b = u / (a.Hkv * f.chunks);
        gh = u / f.chunks - b * a.Hkv;
        chunk = u % f.chunks;
        r = req(b);
        if (chunk >= r.n_chunks) continue;
        unit_base = cost = 0;
        s0 = 0;
        s1 = r.blocks;
      }
      if (s1 <= s0) continue;
      nn = r.nn, kvl = r.kvl, R = r.R, bad = r.bad, cached = r.cached, blocks = r.blocks;
      row0 = chunk * r.rows_each;
      rows = max(0, min(r.rows_each, r.R - row0));
      two = r.rows_each > BM;
      return true;
    }
  }
  __device__ __forceinline__ bool whole() const { return s0 == 0 && s1 == blocks; }
  __device__ __forceinline__ int first_cta() const { return cut.share_of(unit_base + f.unit_cost); }
  __device__ __forceinline__ int last_cta() const {
    return cut.share_of(unit_base + f.unit_cost + (blocks - 1) * (two ? 2 : 1));
  }
  __device__ __forceinline__ int slot(int c) const { return 2 * c + (cut.start(c) < unit_base ? 1 : 0); }
};

__global__ void __launch_bounds__(THREADS, 1) k_kv8_attn_many(const __grid_constant__ CUtensorMap tm_k, ManyArgs f) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  const Kv8Args& a = f.a;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  unsigned char* smem =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sbase = smem_u32(smem);
  const uint32_t sQ = sbase + OFF_Q, sK = sbase + OFF_K, sV = sbase + OFF_V;
  auto bar = [&](int i) { return sbase + OFF_BAR + 8u * (uint32_t)i; };
  if (tid == 0) {
    s_abort = 0;
    for (int i = 0; i < N_BARS; ++i) {
      uint32_t n = 1;
      if (i == B_PFULL || i == B_PFULL + 1) n = 4;
      if (i < B_VEMPTY || (i >= B_QE && i < B_QE + PIECES)) n = NUM_WARPS;
      if (i >= B_QFULL && i < B_QFULL + PIECES) n = NUM_WARPS + 1;
      if (i == B_OFREE || i == B_ML) n = 256;
      mbar_init(bar(i), n);
    }
    fence_mbar_init();
  }
  if (warp == 0) {
    tmem_alloc(smem_u32(&s_tmem), TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  if (warp < 4) regs_dec<REGS_ISSUE>();
  else if (warp >= 12) regs_dec<REGS_NUMBERS>();
  else regs_inc<REGS_SOFTMAX>();
  auto piece = [&](uint32_t i) { return reinterpret_cast<const Piece*>(smem + OFF_PIECE) + i % PIECES; };

  if (warp == 0) {
    // ---------------- products ----------------
    // e4m3 operands: format 0 where bf16 is 1 (bits 7..9, 10..12)
    constexpr uint32_t BF16 = (1u << 7) | (1u << 10);
    constexpr uint32_t IDESC_QK = idesc_bf16_f32(BM, BN, 0) & ~BF16, IDESC_PV = idesc_bf16_f32(BM, HD, 1);
    uint32_t nb = 0, np = 0, t0 = 0, t1 = 0;  // blocks, pieces, steps of each tile so far
    bool ok = true;
    // descriptors' low words: a byte offset adds to them in units of 16
    const uint32_t q_lo = (uint32_t)smem_desc_sw128(sQ, 16, 1024), k_lo = (uint32_t)smem_desc_sw128(sK, 16, 1024);
    const uint32_t k2_lo = (uint32_t)smem_desc_sw128(sbase + OFF_K2, 16, 1024);
    const uint32_t v_lo = (uint32_t)smem_desc_sw128(sV, HALF_BYTES, 1024);
    auto wait = [&](int which, uint32_t parity) {
      ok = ok && warp_wait(bar(which), parity & 1, &s_abort);
      return ok;
    };
    QTile qt;
    for (;;) {
      if (!wait(B_PIECE + np % PIECES, np / PIECES)) break;
      const Piece* pc = piece(np);
      const int n = pc->n;
      if (n == 0) break;
      if (!wait(B_QFULL + np % PIECES, np / PIECES)) break;
      // Steps in order: with two tiles, tile 0 then tile 1 of each block, else
      // the blocks, tile by tile in turn.  Step k's second product comes before
      // step k + 2's first, which writes the scores that P took the place of.
      const int two = pc->two ? 1 : 0, steps = n << two, n_cached = pc->cached - pc->s0;
      qt.next(two);
#pragma unroll 1
      for (int k = -2; k < steps; ++k) {
        const uint32_t x = k & 1;
        const uint32_t blk2 = nb + ((k + 2) >> two);
        if (two && !x && k + 2 < steps && !wait(B_KFULL + blk2 % SLOTS, blk2 / SLOTS)) break;
        if (k >= 0) {  // O_x (+)= P_x V
          const uint32_t blk = nb + (k >> two), st = blk & 1;
          if (!(two & x) && !wait(B_VFULL + st, blk >> 1)) break;  // tile 1: waited for by tile 0
          if (!wait(B_PFULL + x, x ? t1 : t0)) break;
          t0 += 1 - x, t1 += x;
          if (k == 0 && np > 0 && !wait(B_OFREE, np - 1)) break;
          tc_fence_after();
          mma_pv(tmem + 256 + x * 128, tmem + x * 128, v_lo + st * (TILE_BYTES >> 4), IDESC_PV, k >= 2);
          if (!two || x) {
            tc_commit(bar(B_VEMPTY + st));
            tc_commit(bar(B_SLOT + blk % SLOTS));
          }
        }
        if (k + 2 < steps) {  // S_x <- Q K^T
          const uint32_t blk = nb + ((k + 2) >> two), st = blk % SLOTS;
          if (!two && !wait(B_KFULL + st, blk / SLOTS)) break;
          tc_fence_after();
          const uint32_t q1 = q_lo + (two ? x : (uint32_t)qt.tile) * (TILE_BYTES >> 4), q2 = q1 + (HALF_BYTES >> 4);
          const uint32_t k1 = k_lo + st * (HALF_BYTES >> 4), d = tmem + x * 128;
          mma_qk(d, q1, k1, IDESC_QK, 0);
          mma_qk(d, q2, k1, IDESC_QK, 1);
          if ((int)((k + 2) >> two) >= n_cached) {  // new keys have a second part
            mma_qk(d, q1, k2_lo, IDESC_QK, 1);
            mma_qk(d, q2, k2_lo, IDESC_QK, 1);
          }
          tc_commit(bar(B_SFULL + x));
          if (k + 3 == steps) tc_commit(bar(B_QFREE));
        }
      }
      if (!ok) break;
      tc_commit(bar(B_OFIN));
      nb += n;
      ++np;
    }
    if (__any_sync(0xFFFFFFFFu, s_abort)) {  // let issued products retire before the tensor memory is freed
      tc_commit(bar(B_DRAIN));
      volatile int dummy = 0;
      mbar_wait_bounded(bar(B_DRAIN), 0, &dummy, DRAIN_CYCLES);
    }
  } else if (warp < 4) {
    // ---------------- pieces, the list of cut units, padding rows; scales ----------------
    uint32_t np = 0;
    if (warp == 1) {
      Walk wk(f);
      if (f.split && lane == 0) f.list[8 * blockIdx.x] = -1;
      // Description i is written once the queries of piece i - 2 have been
      // used: by then every role is done with piece i - 4, whose place it
      // takes.  Piece i - 1 starts only after this warp has seen that.
      for (;; ++np) {
        if (np >= 2 && !warp_wait(bar(B_QFREE), (np - 2) & 1, &s_abort)) break;
        if (np >= 1 && lane == 0) mbar_arrive(bar(B_QFULL + (np - 1) % PIECES));
        const bool any = wk.next();
        if (lane == 0) {
          Piece* p = reinterpret_cast<Piece*>(smem + OFF_PIECE) + np % PIECES;
          p->n = 0;
          if (any) {
            p->b = wk.b, p->gh = wk.gh, p->row0 = wk.row0, p->rows = wk.rows, p->nn = wk.nn, p->kvl = wk.kvl;
            p->cached = wk.cached, p->s0 = wk.s0, p->n = wk.s1 - wk.s0, p->two = wk.two;
            p->whole = !f.split || wk.whole();
            p->slot = p->whole ? 0 : wk.slot(blockIdx.x);
            if (wk.bad && wk.gh == 0 && wk.s0 == 0 && wk.chunk == 0) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_INVALID);
            if (f.split && wk.s0 > 0 && wk.first_cta() + 1 == (int)blockIdx.x) {  // one entry a cut unit
              const int c0 = blockIdx.x - 1;
              int* e = f.list + 8 * blockIdx.x;
              e[1] = wk.gh, e[2] = wk.row0, e[3] = wk.rows, e[4] = c0, e[5] = wk.last_cta() - c0 + 1;
              e[6] = wk.slot(c0);
              e[0] = wk.b;
            }
          }
          mbar_arrive(bar(B_PIECE + np % PIECES));
        }
        if (!any) break;
        if (wk.s0 == 0 && wk.row0 == 0) {  // the rows past the nodes
          const int pad = (a.n_pad - wk.nn) * a.G;
#pragma unroll 1
          for (int e = lane; e < pad * (HD / 8); e += 32) {
            const int r = e / (HD / 8), ch = e % (HD / 8), i = wk.nn + r / a.G, hh = r % a.G;
            reinterpret_cast<uint4*>(a.out + (((size_t)wk.b * a.n_pad + i) * a.H + wk.gh * a.G + hh) * HD)[ch] =
                make_uint4(0, 0, 0, 0);
          }
        }
      }
    } else if (warp == 2) {
      // ---------------- keys and scales, ahead of the products ----------------
      // Lanes 4i .. 4i + 3: run i (16 keys) of a block's eight.
      const int run_i = lane >> 2, l4 = lane & 3;
      const uint32_t per_page = (uint32_t)a.Hkv << (a.shift - 4), in_page = (1u << (a.shift - 4)) - 1u;
      uint32_t nb = 0, asked = 0;  // blocks; bits of the slots whose last block's keys come by TMA
      bool ok = true;
      for (; ok; ++np) {
        if (!warp_wait(bar(B_PIECE + np % PIECES), (np / PIECES) & 1, &s_abort)) break;
        const Piece pc = *piece(np);
        if (pc.n == 0) break;
        const int s1 = pc.s0 + pc.n, to = min(s1, pc.cached);
        const int32_t* tab = a.table + (size_t)pc.b * a.max_pages;
        auto look_up = [&](int blk) {
          const uint32_t run = (uint32_t)blk * (BN / 16) + run_i;
          return blk < to && run <= (uint32_t)(pc.kvl - 1) >> 4 ? tab[run >> (a.shift - 4)] : -1;
        };
        int id = look_up(pc.s0), id_next = look_up(pc.s0 + 1);
        uint32_t run = 0;
        float ks = 0.f, vs = 0.f;
        bool in = false;
        auto fetch = [&](int blk) {
          in = (unsigned)id < (unsigned)a.n_pages;
          run = in ? id * per_page + ((uint32_t)pc.gh << (a.shift - 4)) + (((uint32_t)blk * (BN / 16) + run_i) & in_page) : 0u;
          ks = a.ks[run];
          vs = a.vs[run];
          // the values' rows, asked into L2
#pragma unroll
          for (int u = 0; u < 4; ++u) prefetch_l2(a.vc + (uint64_t)run * 2048u + (l4 + 4 * u) * 128);
        };
        if (pc.s0 < to) fetch(pc.s0);
        for (int blk = pc.s0; blk < s1; ++blk, ++nb) {
          const int slot = nb % SLOTS;
          const bool fresh = blk >= pc.cached;
          const uint32_t run_now = run;
          int left;  // keys of the run that count
          float back = 1.f, mul = 0.f;
          if (!fresh) {
            const long long more = pc.kvl - ((long long)blk * BN + 16 * run_i);
            left = in ? (int)min(16ll, max(0ll, more)) : 0;
            if (!in && more > 0 && l4 == 0) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_INVALID);
            back = left ? ks : 1.f;  // whatever stands where no key counts
            mul = left ? vs : 0.f;
            if (blk + 1 < to) {
              id = id_next;
              fetch(blk + 1);
              id_next = look_up(blk + 2);
            }
          } else {
            left = a.k_new ? min(16, max(0, pc.nn - 16 * run_i)) : 0;  // (their factors: by the warps that split them)
          }
          if (nb >= SLOTS && !(ok = warp_wait(bar(B_SLOT + slot), (nb / SLOTS - 1) & 1, &s_abort))) break;
          if (l4 == 0) {
            reinterpret_cast<uint16_t*>(smem + OFF_KEEP + slot * 16)[run_i] = (uint16_t)((1u << left) - 1u);
            reinterpret_cast<float*>(smem + OFF_BACK)[slot * (BN / 16) + run_i] = back;
            reinterpret_cast<float*>(smem + OFF_VS)[slot * (BN / 16) + run_i] = mul;
            reinterpret_cast<uint32_t*>(smem + OFF_RUN)[slot * (BN / 16) + run_i] = run_now;
            if (!fresh) {
              mbar_expect_tx(bar(B_KFULL + slot), 2048);
              tma_load_3d(sK + slot * HALF_BYTES + run_i * 2048, &tm_k, 0, 0, (int)run_now, bar(B_KFULL + slot));
            }
          }
          asked = fresh ? asked & ~(1u << slot) : asked | (1u << slot);
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(B_INFO + slot));
        }
      }
      if (__any_sync(0xFFFFFFFFu, s_abort)) {  // let the copies in flight land before the CTA exits
        volatile int dummy = 0;
        for (uint32_t i = nb > SLOTS ? nb - SLOTS : 0; i < nb; ++i)
          if ((asked >> (i % SLOTS)) & 1u) mbar_wait_bounded(bar(B_KFULL + i % SLOTS), (i / SLOTS) & 1, &dummy, DRAIN_CYCLES);
      }
    }
  } else if (warp >= 12) {
    // ---------------- queries and values to tiles ----------------
    // Warp w has rows 16w .. 16w + 15 of a block, one run of a page: lane (rho,
    // c) rows rho and rho + 8, dimensions 32c .. 32c + 31.  Eight lanes in turn have
    // eight rows, so that their stores fall in different banks.
    // Column 8i + 2q + e of 32 is dimension 8q + 2i + e: so a thread that reads the
    // sums back, columns 2q and 2q + 1 of every 8, has 8 dimensions that are neighbours.
    const int w = warp - 12, c = lane >> 3, rho = lane & 7;
    const uint32_t dst = (c >> 1) * HALF_BYTES + (16 * w + rho) * 128 + ((((c & 1) * 4) ^ rho) << 4);
    Piece pc = {};
    uint4 vr[4];  // row rho, then row rho + 8
    uint32_t nb = 0;
    bool ok = true;
    auto info = [&](uint32_t blk) {
      return warp_wait(bar(B_INFO + blk % SLOTS), (blk / SLOTS) & 1, &s_abort);
    };
    const uint32_t* runs = reinterpret_cast<const uint32_t*>(smem + OFF_RUN) + w;
    const float* vscales = reinterpret_cast<const float*>(smem + OFF_VS) + w;
    auto fetch = [&](uint32_t run) {
      const uint8_t* src = a.vc + (uint64_t)run * 2048u + rho * 128 + 32 * c;
      ld_global32(vr[0], vr[1], src);
      ld_global32(vr[2], vr[3], src + 8 * 128);
    };
    // The piece's queries, a row 16 lanes: all of them asked for at once, a chunk of
    // 8 values in two halves, each where a part of the chunk will be.  Rows past
    // the last 32 of which some are in use are not written.
    auto stage_q = [&](uint32_t np, int tile) {
      const int ch = lane & 15, r0 = 2 * w + (lane >> 4), passes = ((pc.rows + 31) >> 5) * 2;  // 16 rows each
      const uint32_t to0 = OFF_Q + tile * TILE_BYTES + r0 * 128 + (((ch >> 1) ^ (r0 & 7)) << 4) + (ch & 1) * 8;
      auto at = [&](int p) { return to0 + p * 2048 + (p & 8) * 2048; };  // the second tile from pass 8 on
      const __nv_bfloat16* q0 = a.q + ((size_t)pc.b * a.n_pad * a.H + pc.gh * a.G) * HD + ch * 8;
#pragma unroll 1
      for (int p = 0; p < passes; ++p) {
        const uint32_t to = sbase + at(p);
        const int r = r0 + 16 * p, rr = pc.row0 + r;
        if (r < pc.rows) {
          const __nv_bfloat16* src = q0 + (size_t)(uint32_t)(f.node_of(rr) * (a.H - a.G) + rr) * HD;
          cp_async8(to, src);
          cp_async8(to + HALF_BYTES, src + 4);
        } else {
          unsigned char* z = smem + at(p);
          *reinterpret_cast<uint2*>(z) = *reinterpret_cast<uint2*>(z + HALF_BYTES) = make_uint2(0, 0);
        }
      }
      cp_async_wait_all();
      float* back = reinterpret_cast<float*>(smem + OFF_QE) + np % PIECES * ROWS + r0;
#pragma unroll 1
      for (int p0 = 0; p0 < passes; p0 += QN) {
        uint2 lo[QN], hi[QN];
        uint32_t top[QN];
#pragma unroll
        for (int k = 0; k < QN; ++k) {
          const unsigned char* from = smem + at(p0 + k);
          lo[k] = *reinterpret_cast<const uint2*>(from);
          hi[k] = *reinterpret_cast<const uint2*>(from + HALF_BYTES);
          const uint32_t sign = 0x7FFF7FFFu;
          top[k] = __vmaxu2(__vmaxu2(lo[k].x & sign, lo[k].y & sign), __vmaxu2(hi[k].x & sign, hi[k].y & sign));
        }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1)
#pragma unroll
          for (int k = 0; k < QN; ++k) top[k] = __vmaxu2(top[k], __shfl_xor_sync(0xFFFFFFFFu, top[k], o));
#pragma unroll
        for (int k = 0; k < QN; ++k) {
          const int ex = expo_of(max(top[k] & 0xFFFFu, top[k] >> 16));
          if (ch == 0) back[16 * (p0 + k)] = pow2i(ex - E_TOP);
          uint2 p1, p2;
          split8(make_uint4(lo[k].x, lo[k].y, hi[k].x, hi[k].y), pow2i(E_TOP - ex), p1, p2);
          unsigned char* to = smem + at(p0 + k);
          *reinterpret_cast<uint2*>(to) = p1;
          *reinterpret_cast<uint2*>(to + HALF_BYTES) = p2;
        }
      }
    };
    auto done = [&](int which) {  // this warp's part of a tile is written
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(which));
    };
    QTile qt;
    for (uint32_t np = 0; ok; ++np) {
      if (!warp_wait(bar(B_PIECE + np % PIECES), (np / PIECES) & 1, &s_abort)) break;
      pc = *piece(np);
      if (pc.n == 0) break;
      const int s1 = pc.s0 + pc.n;
      uint32_t run = 0;
      if (pc.s0 < pc.cached) {
        if (!(ok = info(nb))) break;
        run = runs[nb % SLOTS * (BN / 16)];
        fetch(run);
      }
      if (qt.next(pc.two) && np > 0 && !(ok = warp_wait(bar(B_QFREE), (np - 1) & 1, &s_abort))) break;
      stage_q(np, qt.tile);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar(B_QE + np % PIECES));
        mbar_arrive(bar(B_QFULL + np % PIECES));
      }
      const int to = min(s1, pc.cached);
#pragma unroll 1
      for (int blk = pc.s0; blk < to; ++blk, ++nb) {
        const int st = nb & 1, slot = nb % SLOTS;
        const bool more = blk + 1 < to;
        // 2^120 times the scale, in two factors that bf16 holds
        const float s = vscales[slot * (BN / 16)];
        const int ex = min(max(kv8_exp(s), KV8_MIN_EXP), KV8_MAX_EXP) + 120, e1 = min(ex, 127);
        const float m1 = kv8_nan(s) || s == 0.f ? s : pow2i(e1);
        const uint32_t f1 = pack_bf16x2(m1, m1), f2 = pack_bf16x2(pow2i(ex - e1), pow2i(ex - e1));
        if (nb >= 2 && !(ok = warp_wait(bar(B_VEMPTY + st), ((nb >> 1) - 1) & 1, &s_abort))) break;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          unsigned char* t = smem + OFF_V + st * TILE_BYTES + k * 1024;
          const uint4 a0 = vr[2 * k], a1 = vr[2 * k + 1];
          *reinterpret_cast<uint4*>(t + dst) = values8(a0.x, a0.z, a1.x, a1.z, 0x1000, f1, f2);
          *reinterpret_cast<uint4*>(t + (dst ^ 16)) = values8(a0.x, a0.z, a1.x, a1.z, 0x3020, f1, f2);
          *reinterpret_cast<uint4*>(t + (dst ^ 32)) = values8(a0.y, a0.w, a1.y, a1.w, 0x1000, f1, f2);
          *reinterpret_cast<uint4*>(t + (dst ^ 48)) = values8(a0.y, a0.w, a1.y, a1.w, 0x3020, f1, f2);
        }
        done(B_VFULL + st);
        if (more) {
          if (!(ok = info(nb + 1))) break;
          run = runs[(nb + 1) % SLOTS * (BN / 16)];
          fetch(run);
        }
      }
      if (ok && to < s1) {  // the new tokens' block
        const int st = nb & 1, slot = nb % SLOTS;
        if (!(ok = info(nb))) break;
        // the second part's place: free once the last piece's first products are done
        if (np > 0 && !(ok = warp_wait(bar(B_QFREE), (np - 1) & 1, &s_abort))) break;
        // rows 16w .. of the new tokens; keys' halves where their parts will be, values in their place
        const int live = a.k_new ? min(16, pc.nn - 16 * w) : 0;
        const size_t from = (((size_t)pc.b * a.Hkv + pc.gh) * a.n_pad + 16 * w) * HD;
        const uint32_t sK1 = OFF_K + slot * HALF_BYTES, ch = lane & 15;
        const uint32_t k0 = (16 * w + (lane >> 4)) * 128 + (((ch >> 1) ^ (lane >> 4)) << 4) + (ch & 1) * 8;
        auto k_at = [&](int j) { return (k0 ^ ((j & 6) << 4)) + (j >> 1) * 256; };  // of row j, lane >> 4 in its lowest bit
        const uint32_t sV1 = OFF_V + st * TILE_BYTES + (ch >> 3) * HALF_BYTES;
        auto v_at = [&](int j, int i) { return sV1 + (16 * w + j) * 128 + (((ch & 4) ^ i ^ (j & 7)) << 4); };
#pragma unroll 1
        for (int j = lane >> 4; j < live; j += 2) {
          cp_async8(sbase + sK1 + k_at(j), a.k_new + from + j * HD + ch * 8);
          cp_async8(sbase + OFF_K2 + k_at(j), a.k_new + from + j * HD + ch * 8 + 4);
        }
        cp_async_commit();
        if (nb >= 2 && !(ok = warp_wait(bar(B_VEMPTY + st), ((nb >> 1) - 1) & 1, &s_abort))) break;
#pragma unroll 1
        for (int j = lane >> 4; j < 16; j += 2) {
          if (j < live) cp_async16(sbase + v_at(j, ch & 3), a.v_new + from + j * HD + ch * 8);
          else *reinterpret_cast<uint4*>(smem + v_at(j, ch & 3)) = make_uint4(0, 0, 0, 0);
        }
        cp_async_commit();
        cp_async_wait<1>();
        uint32_t top = 0;
#pragma unroll 1
        for (int j = lane >> 4; j < live; j += 2) {
          const uint2 lo = *reinterpret_cast<const uint2*>(smem + sK1 + k_at(j)), hi = *reinterpret_cast<const uint2*>(smem + OFF_K2 + k_at(j));
          top = top2(top2(top2(top2(top, lo.x), lo.y), hi.x), hi.y);
        }
        const int ek = expo_of(__reduce_max_sync(0xFFFFFFFFu, max(top & 0xFFFFu, top >> 16)));
        if (lane == 0) reinterpret_cast<float*>(smem + OFF_BACK)[slot * (BN / 16) + w] = pow2i(ek - E_TOP);
#pragma unroll 1
        for (int j = lane >> 4; j < live; j += 2) {
          uint2 *k1 = reinterpret_cast<uint2*>(smem + sK1 + k_at(j)), *k2 = reinterpret_cast<uint2*>(smem + OFF_K2 + k_at(j));
          const uint2 lo = *k1, hi = *k2;
          split8(make_uint4(lo.x, lo.y, hi.x, hi.y), pow2i(E_TOP - ek), *k1, *k2);
        }
        done(B_KFULL + slot);
        cp_async_wait<0>();
        __syncwarp();
        // Into their columns: four lanes exchange the words of 32 dimensions.  A
        // value that is not finite becomes 0, as no weight of 0 would take it
        // out of the rows that do not see its token; those that do are NaN.
        uint32_t bad = 0;
#pragma unroll 1
        for (int j = lane >> 4; j - (lane >> 4) < live; j += 2) {
          const uint4 v = *reinterpret_cast<const uint4*>(smem + v_at(j, ch & 3));
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t x = (&v.x)[i], not_finite = __vcmpgeu2(x & 0x7FFF7FFFu, 0x7F807F80u);
            *reinterpret_cast<uint32_t*>(smem + v_at(j, i) + (ch & 3) * 4) = x & ~not_finite;
            if (not_finite) bad |= 1u << j;
          }
        }
        bad = __reduce_or_sync(0xFFFFFFFFu, bad);
        if (lane == 0) reinterpret_cast<uint16_t*>(smem + OFF_BAD)[np % PIECES * NUM_WARPS + w] = (uint16_t)bad;
        done(B_VFULL + st);
        ++nb;
      }
    }
    cp_async_wait_all();
  } else {
    // ---------------- softmax: warpgroup x, a row a thread ----------------
    // (A piece's description is read again where it is needed, not kept: the
    // loop wants its registers for the scores.)
    const int x = (warp - 4) >> 2, r = (warp & 3) * 32 + lane;
    const uint32_t tS = tmem + x * 128 + ((uint32_t)((warp & 3) * 32) << 16), tO = tS + 256;
    uint32_t nb = 0, np = 0, nx = 0, t = 0;
    bool ok = true;
    auto row_of = [&](const Piece* pc) { return pc->two ? x * BM + r : r; };  // row of the piece
    auto seen = [&](const Piece* pc, uint64_t (&sees)[2]) {  // the new tokens that the row sees
      const int lr = row_of(pc), i = f.node_of(pc->row0 + lr);
      if (lr >= pc->rows) {
        sees[0] = sees[1] = 0;
      } else if (a.mask) {
        const int words = (a.n_pad + 63) / 64;
        const uint64_t* mr = a.mask + ((size_t)pc->b * a.n_pad + i) * words;
        sees[0] = mr[0];
        sees[1] = words > 1 ? mr[1] : 0ull;
      } else {
        sees[0] = i >= 63 ? ~0ull : (1ull << (i + 1)) - 1ull;
        sees[1] = i < 64 ? 0ull : (i >= 127 ? ~0ull : (1ull << (i - 63)) - 1ull);
      }
    };
    for (;;) {
      if (!(ok = warp_wait(bar(B_PIECE + np % PIECES), (np / PIECES) & 1, &s_abort))) break;
      const Piece* pc = piece(np);
      const int n = pc->n;
      if (n == 0) break;
      float m = M_START, l = 0.f;  // m: the reference
      if (!(ok = warp_wait(bar(B_QE + np % PIECES), (np / PIECES) & 1, &s_abort))) break;
      const float c_row =
          fminf(fmaxf(a.scale_log2 * reinterpret_cast<const float*>(smem + OFF_QE)[np % PIECES * ROWS + row_of(pc)], ROW_MIN), FACTOR_MAX);
      const int every = pc->two ? 1 : 2, first = pc->two ? 0 : x, n_cached = pc->cached - pc->s0;
      const bool idle = row_of(pc) - lane >= pc->rows;  // none of the warp's rows is in use
#pragma unroll 1
      for (int j = first; j < n; j += every, ++t) {
        if (idle) {
          if (!(ok = warp_wait(bar(B_SFULL + x), t & 1, &s_abort))) break;
          if (lane == 0) mbar_arrive(bar(B_PFULL + x));
          continue;
        }
        const int slot = (nb + j) % SLOTS;
        if (!(ok = warp_wait(bar(B_INFO + slot), ((nb + j) / SLOTS) & 1, &s_abort))) break;
        const float2* back = reinterpret_cast<const float2*>(smem + OFF_BACK) + slot * (NUM_WARPS / 2);
        const uint32_t* keep = reinterpret_cast<const uint32_t*>(smem + OFF_KEEP) + slot * 4;
        const bool masked = j >= n_cached || (keep[0] & keep[1] & keep[2] & keep[3]) != 0xFFFFFFFFu;  // in all rows alike
        uint64_t sees[2] = {~0ull, ~0ull};
        if (j >= n_cached) {
          seen(pc, sees);
          // the new keys' factors come with the keys
          if (!(ok = warp_wait(bar(B_KFULL + slot), ((nb + j) / SLOTS) & 1, &s_abort))) break;
        }
        if (!(ok = warp_wait(bar(B_SFULL + x), t & 1, &s_abort))) break;
        tc_fence_after();
        if (__builtin_expect(masked, 0)) {  // masked scores are overwritten by -inf
#pragma unroll 1
          for (int q = 0; q < 4; ++q) {
            const uint32_t k = keep[q] & (uint32_t)(sees[q >> 1] >> (32 * (q & 1)));
            uint32_t sv[32];
            tmem_ld32(tS + q * 32, sv);
            tc_wait_ld();
#pragma unroll
            for (int u = 0; u < 32; ++u)
              if (!((k >> u) & 1u)) sv[u] = __float_as_uint(-INFINITY);
            tmem_st32(tS + q * 32, sv);
          }
          tc_wait_st();
        }
        // The row's scores come 32 at a time, once for the maximum, once for P, one
        // short loop each: the roles share the instruction cache, and the other
        // warps cover the loads.  (64 at a time, at a step where this took 893 us for
        // 32 trees of 128 nodes and 121 for 16 of 64: 880 and 129.)
        uint32_t sa[32], sb[32];
        float top = -INFINITY;
        auto largest = [&](int q, const uint32_t (&sv)[32]) {
          const float2 bk = back[q];  // of its two runs of 16 keys
          float p0 = -INFINITY, p1 = -INFINITY;
#pragma unroll
          for (int u = 0; u < 16; u += 2) {
            p0 = max3(p0, __uint_as_float(sv[u]), __uint_as_float(sv[u + 1]));
            p1 = max3(p1, __uint_as_float(sv[16 + u]), __uint_as_float(sv[17 + u]));
          }
          top = max3(top, p0 * bk.x, p1 * bk.y);
        };
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          tmem_ld32(tS + q * 32, sa);
          tc_wait_ld();
          largest(q, sa);
        }
        {
          top *= c_row;
          if (__builtin_expect(__any_sync(0xFFFFFFFFu, top > m + RESCALE_THRESHOLD), 0)) {
            const float m_new = top > m + RESCALE_THRESHOLD ? top : m, alpha = exp2_fast(m - m_new);
            l *= alpha;
            m = m_new;
            if (j > first) {  // S_x is the newest product of this tile, so O_x is complete
#pragma unroll 1
              for (int cc = 0; cc < HD / 32; ++cc) {
                tmem_ld32(tO + cc * 32, sb);
                tc_wait_ld();
#pragma unroll
                for (int u = 0; u < 32; ++u) sb[u] = __float_as_uint(__uint_as_float(sb[u]) * alpha);
                tmem_st32(tO + cc * 32, sb);
              }
            }
          }
        }
        uint64_t sum[2] = {0ull, 0ull};
        const uint64_t neg = f2_pack(-m, -m);
        auto weigh = [&](int q, const uint32_t (&sv)[32]) {  // over scores already read
          uint32_t pk[16];
          const float2 bk = back[q];
#pragma unroll
          for (int u = 0; u < 16; ++u) {
            const float cz = min_nan(max_nan(c_row * (u < 8 ? bk.x : bk.y), FACTOR_MIN), FACTOR_MAX);
            float p0, p1;
            f2_unpack(f2_fma(f2_pack(__uint_as_float(sv[2 * u]), __uint_as_float(sv[2 * u + 1])), f2_pack(cz, cz), neg), p0, p1);
            p0 = exp2_fast(p0), p1 = exp2_fast(p1);
            sum[u & 1] = f2_add(sum[u & 1], f2_pack(p0, p1));
            pk[u] = pack_bf16x2(p0, p1);
          }
          tmem_st16(tS + q * 16, pk);
        };
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          tmem_ld32(tS + q * 32, sa);
          tc_wait_ld();
          weigh(q, sa);
        }
        tc_wait_st();
        float s0, s1;
        f2_unpack(f2_add(sum[0], sum[1]), s0, s1);
        l += s0 + s1;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_PFULL + x));
      }
      if (!ok || !(ok = warp_wait(bar(B_OFIN), np & 1, &s_abort))) break;
      tc_fence_after();
      // ---- the piece's rows: this tile's, or half the dimensions of both halves' sum
      const bool two = pc->two, whole = pc->whole;
      if (n > n_cached) {  // new tokens: are all values finite?
        const uint64_t* bad = reinterpret_cast<const uint64_t*>(smem + OFF_BAD) + np % PIECES * 2;
        if (bad[0] | bad[1]) {
          uint64_t sees[2];
          seen(pc, sees);
          if ((sees[0] & bad[0]) | (sees[1] & bad[1])) l = __uint_as_float(0x7FC00000u);
        }
      }
      float m_all = m, k0 = 1.f, k1 = 0.f;
      uint32_t tO0 = tO;
      if (!two) {
        // two turns' room: a turn is written again only after both have read it
        float2* ml = reinterpret_cast<float2*>(smem + OFF_ML) + (nx & 1) * 2 * BM;
        ml[x * BM + r] = make_float2(m, l);
        mbar_arrive(bar(B_ML));
        if (!(ok = warp_wait(bar(B_ML), nx & 1, &s_abort))) break;
        ++nx;
        const float2 other = ml[(1 - x) * BM + r];
        m_all = fmaxf(m, other.x);
        const float mine = exp2_fast(m - m_all), theirs = exp2_fast(other.x - m_all);
        l = l * mine + other.y * theirs;
        k0 = x == 0 ? mine : theirs;
        k1 = x == 0 ? theirs : mine;
        tO0 -= x * 128;
      }
      const float inv = !whole ? 1.f : (l == 0.f ? 0.f : 1.f / l);
      k0 *= inv;
      k1 *= inv;
      const bool both = !two && n > 1;
      const int row_w = row_of(pc) - lane;  // the warp's first row
      const size_t slot0 = (size_t)pc->slot * f.rows_cap;
      // 16 rows and 32 dimensions at a time: a lane has 8 neighbours of two rows, four lanes 64 (a lane a row,
      // its stores in 32 rows each, took 7000 cycles for 256 rows, this 3000)
#pragma unroll 1
      for (int half = idle ? 32 : 0; half < 32; half += 16) {
        float ka[2], kb[2];
        bool in[2];
        __nv_bfloat16* dst[2];
        float* po[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int from = half + 8 * k + (lane >> 2), lr = row_w + from, rr = pc->row0 + lr;
          ka[k] = __shfl_sync(0xFFFFFFFFu, k0, from);
          kb[k] = __shfl_sync(0xFFFFFFFFu, k1, from);
          in[k] = lr < pc->rows;
          dst[k] = a.out + ((size_t)(uint32_t)(f.node_of(rr) * (a.H - a.G) + rr) + (size_t)pc->b * a.n_pad * a.H + pc->gh * a.G) * HD + (lane & 3) * 8;
          po[k] = f.part_o + (slot0 + lr) * HD + (lane & 3) * 8;
        }
#pragma unroll 1
        for (int cc = two ? 0 : 2 * x; cc < (two ? 4 : 2 * x + 2); ++cc) {
          uint32_t o[16], o2[16];
          tmem_ld_rows(tO0 + (half << 16) + cc * 32, o);
          if (both) tmem_ld_rows(tO0 + (half << 16) + 128 + cc * 32, o2);
          tc_wait_ld();
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const int i = 4 * (u >> 1) + 2 * k + (u & 1);
              v[u] = __uint_as_float(o[i]) * ka[k];
              if (both) v[u] = fmaf(__uint_as_float(o2[i]), kb[k], v[u]);
            }
            if (!in[k]) continue;
            if (whole) {
              *reinterpret_cast<uint4*>(dst[k] + cc * 32) =
                  make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
            } else {
              float4* p = reinterpret_cast<float4*>(po[k] + cc * 32);
              p[0] = make_float4(v[0], v[1], v[2], v[3]);
              p[1] = make_float4(v[4], v[5], v[6], v[7]);
            }
          }
        }
      }
      if (!whole && row_w + lane < pc->rows && (two || x == 0)) f.part_ml[slot0 + row_w + lane] = make_float2(m_all, l);
      tc_fence_before();
      mbar_arrive(bar(B_OFREE));
      nb += n;
      ++np;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && s_abort) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_TIMEOUT);
  if (warp == 0) {
    tc_fence_after();
    tmem_dealloc(tmem, TMEM_COLS);
  }
}

// The pieces of cut units, added up in CTA order.  CTA (c, y): the unit whose
// second piece CTA c of k_kv8_attn_many began with, 8 of its rows, a warp each.
__global__ void __launch_bounds__(256) k_kv8_join(ManyArgs f) {
  const Kv8Args& a = f.a;
  const int* e = f.list + 8 * blockIdx.x;
  const int b = e[0];
  if (b < 0) return;
  const int gh = e[1], row0 = e[2], rows = e[3], c0 = e[4], nc = e[5], slot0 = e[6];
  const int lane = threadIdx.x & 31, r = blockIdx.y * 8 + (threadIdx.x >> 5);
  if (r >= rows) return;
  auto slot = [&](int c) { return (size_t)(c == 0 ? slot0 : 2 * (c0 + c)) * f.rows_cap + r; };
  float m = -INFINITY;
  for (int c = lane; c < nc; c += 32) m = fmaxf(m, f.part_ml[slot(c)].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  if (m == -INFINITY) m = 0.f;
  float l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int c = 0; c < nc; ++c) {
    const float2 ml = f.part_ml[slot(c)];
    const float4 v = reinterpret_cast<const float4*>(f.part_o + slot(c) * HD)[lane];
    const float k = exp2_fast(ml.x - m);
    l += ml.y * k;
    acc.x += v.x * k, acc.y += v.y * k, acc.z += v.z * k, acc.w += v.w * k;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int i = f.node_of(row0 + r), hh = row0 + r - i * a.G;
  __nv_bfloat16* dst = a.out + (((size_t)b * a.n_pad + i) * a.H + gh * a.G + hh) * HD + 4 * lane;
  *reinterpret_cast<uint2*>(dst) =
      make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
}

int rows_of_chunk(int n_pad, int G) { return std::min(ROWS, n_pad * G); }

size_t list_bytes(int grid) { return ((size_t)grid * 32 + 255) / 256 * 256; }
size_t slot_bytes(int rows) { return (size_t)rows * (HD * sizeof(float) + sizeof(float2)); }

constexpr int FULL_GRID = 152;

PFN_cuTensorMapEncodeTiled_v12000 get_encode() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  });
  return fn;
}

// The keys as runs of 16 rows of 128 bytes; a box is a run, 128-byte swizzle.
bool make_map(CUtensorMap* m, const Kv8Args& a) {
  auto enc = get_encode();
  if (!enc) return false;
  cuuint64_t dims[3] = {HD, 16, ((cuuint64_t)a.n_pages * a.Hkv) << (a.shift - 4)};
  cuuint64_t strides[2] = {HD, 16 * HD};
  cuuint32_t box[3] = {HD, 16, 1}, es[3] = {1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<uint8_t*>(a.kc), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

size_t kv8_attn_many_workspace(int batch, int n_pad, int H, int Hkv) {
  (void)batch;
  return KV8_WS_COUNTERS + list_bytes(FULL_GRID) + (size_t)FULL_GRID * 2 * slot_bytes(rows_of_chunk(n_pad, H / Hkv));
}

fc_status kv8_attn_many(const Kv8Args& a, void* ws, size_t ws_bytes, cudaStream_t s) {
  static std::atomic<unsigned long long> done{0};
  const fc_status st = fc_once_per_device(done, [](int) {
    cudaFuncAttributes attr;
    if (cudaFuncGetAttributes(&attr, k_kv8_attn_many) != cudaSuccess) return FC_ERR_CUDA;
    if (attr.numRegs < REGS_LAUNCH) return FC_ERR_INTERNAL;  // the register split would not add up
    return fc_cuda_status(cudaFuncSetAttribute(k_kv8_attn_many, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES));
  });
  if (st != FC_OK) return st;
  ManyArgs f{a, 0, 1, CUT_COST, rows_of_chunk(a.n_pad, a.G), ((1u << 20) + a.G - 1) / a.G, nullptr, nullptr, nullptr};
  f.chunks = (a.n_pad * a.G + ROWS - 1) / ROWS;
  const long long units = (long long)a.B * a.Hkv * f.chunks;
  if (units > 0x7FFFFFFFll) return FC_ERR_UNSUPPORTED;
  if (units > 2 * FULL_GRID) f.unit_cost = WHOLE_COST;
  const long long longest = (((long long)a.max_pages << a.shift) + BN - 1) / BN + 1;
  const bool fits = units * (WHOLE_COST + 2 * longest) <= 0x7FFFFFFFll;
  int grid = (int)std::min<long long>(FULL_GRID, units * ((CUT_COST + 2 * longest) / LEAST));
  auto need = [&] { return KV8_WS_COUNTERS + list_bytes(grid) + (size_t)grid * 2 * slot_bytes(f.rows_cap); };
  while (grid > 1 && ws && need() > ws_bytes) --grid;
  // a workspace for fewer CTAs than whole units would fill: whole units
  if (!ws || !fits || need() > ws_bytes || grid < std::min<long long>(FULL_GRID, units)) {
    f.split = 0;
    grid = (int)std::min<long long>(units, FULL_GRID);
  } else {
    unsigned char* p = static_cast<unsigned char*>(ws) + KV8_WS_COUNTERS;
    f.list = reinterpret_cast<int*>(p);
    f.part_o = reinterpret_cast<float*>(p + list_bytes(grid));
    f.part_ml = reinterpret_cast<float2*>(f.part_o + (size_t)grid * 2 * f.rows_cap * HD);
  }
  CUtensorMap tm_k;
  if (!make_map(&tm_k, a)) return FC_ERR_CUDA;
  k_kv8_attn_many<<<grid, THREADS, SMEM_BYTES, s>>>(tm_k, f);
  if (f.split && grid > 1) k_kv8_join<<<dim3(grid, (f.rows_cap + 7) / 8), 256, 0, s>>>(f);
  return FC_CHECK_LAUNCH();
}
