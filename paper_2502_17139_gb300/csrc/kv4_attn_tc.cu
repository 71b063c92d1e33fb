// fc_kv4_attn for more than 16 query rows a kv head (draft trees, chunks): the
// tensor cores' products over the paged 4-bit cache.
//
// A unit is up to 256 query rows of one (sequence, kv head) and all its keys,
// in blocks of 128 keys, the new tokens the last.  Per block
//   S = Q K^T,  P = 2^(c S - m) * (value scale),  O += P V.
// The first product is in fp16: a cached key's values c * s have at most 3 + 8
// significant bits, so they are exact, and powers of two (one per query row,
// one per 16 keys) keep them in range.  The second is in bf16, P needing
// its range: V the whole numbers -7..7, their scales multiplied into P.
// (Folding these into V as well would round them; applying K's scales to S
// would have every row read them from shared memory, as it does V's.)
//   * Two warps look the pages up, ask the rows into L2 and work the scales out,
//     up to four blocks ahead.
//   * Eight warps turn 4-bit rows into 16-bit tiles in shared memory (128-byte
//     swizzle), two stages of K and V each, one block ahead in registers.  A
//     number c + 8 placed in bits 6..9 of a half is 16 + (c + 8) in fp16; one
//     packed fma with (s, -24 s), exact, makes it c s.  In bits 0..3 it is 128
//     + (c + 8) in bf16, and one subtraction makes it c.  A word's 8 numbers come out
//     as the pairs (0,4) (1,5) (2,6) (3,7), so dimensions are kept in that
//     order within groups of 8: queries and the new tokens' rows are put in
//     it, the output taken out of it.
//   * One warp issues every tcgen05.mma (accumulators and P in tensor memory).
//   * Two softmax warpgroups, a row a thread.  With more than 128 rows each has
//     its tile and both take every block; with fewer both have the same rows,
//     one takes the even blocks and one the odd, and their halves are joined
//     at the end, so that one tile's softmax always has the other's products
//     beside it.
//   * The eight warps also fetch a unit's queries, while the last one's end is
//     written.
// The CTAs (one an SM) share all units' blocks equally, cut anywhere; a cut
// unit's pieces go through the workspace to k_kv4_join.
// Measured (kv heads x their query heads): 32 trees of 128 nodes over 16384 keys
// (8 x 4) 1070 us, 1028 TFLOP/s of the tree's own products; 16 trees of 64 nodes
// over 4096 (32 x 1) 217 us; one of 128 over 500 keys 35 us.  With two tiles a
// block takes 4.1 K cycles: 2.6 K of softmax, then the 1.1 K of that tile's two
// products, waits the rest; the other tile runs beside it.  With one tile it
// takes 3.5 K, where the two stages of K and V tie a block to the products of
// the two before; no part alone bounds that (0.91 of the time without
// conversion, 0.86 without softmax, 0.78 without both).
// Several roles run at once from one instruction cache, so the loops are short:
// unrolling or doubling one body for latency's sake cost 3 to 10%.
// Every mbarrier wait is bounded: one that runs out raises FC_ERR_TIMEOUT, the
// CTA lets its issued products retire, frees its tensor memory and returns.
#include <algorithm>
#include <atomic>

#include "fc_common.cuh"
#include "kv4.cuh"

FC_DEFINE_ERROR_WORD(kv4_tc)

namespace {

constexpr int HD = KV4_D;
constexpr int THREADS = 640;  // warp 0 products, 1 pieces, 2-3 scales, 4-7 / 8-11 softmax, 12-19 queries and numbers to tiles
constexpr int NUM_WARPS = 8;
constexpr int BM = 128, BN = 128, ROWS = 2 * BM;
constexpr uint32_t HALF_BYTES = 128 * 128;         // 64 dims of 128 rows
constexpr uint32_t TILE_BYTES = 2 * HALF_BYTES;
constexpr uint32_t OFF_Q = 0;                      // two tiles
constexpr uint32_t OFF_K = OFF_Q + 2 * TILE_BYTES; // two stages
constexpr uint32_t OFF_V = OFF_K + 2 * TILE_BYTES;
constexpr int SLOTS = 4;                                        // blocks whose scales and keep bits are kept
constexpr uint32_t OFF_KEEP = OFF_V + 2 * TILE_BYTES;           // [slot][4] bits of the keys that count
constexpr uint32_t OFF_VS = OFF_KEEP + SLOTS * 16;              // [slot][128] value scales, bf16
constexpr uint32_t OFF_BACK = OFF_VS + SLOTS * BN * 4;          // [slot][8] what 16 keys' scores are to be multiplied by
constexpr uint32_t OFF_RUN = OFF_BACK + SLOTS * 32;             // [slot][8] where 16 keys' rows are, in runs of 16 rows
constexpr uint32_t OFF_KS = OFF_RUN + SLOTS * 32;               // [slot][128] (s, s), (-24 s, -24 s): a key's scale in fp16
constexpr int PIECES = 4;                                       // piece descriptions kept
constexpr uint32_t OFF_QE = OFF_KS + SLOTS * BN * 8;            // [PIECES][256] what a query row's scores are to be multiplied by
constexpr uint32_t OFF_ML = OFF_QE + PIECES * ROWS * 4;              // [2 turns][2][128] (m, l) exchanged at a unit's end
constexpr uint32_t OFF_BAD = OFF_ML + 4 * BM * 8;               // [PIECES][8] bits of the new tokens whose values are not finite
constexpr uint32_t OFF_PIECE = OFF_BAD + PIECES * 16;           // [PIECES]
constexpr uint32_t OFF_BAR = OFF_PIECE + PIECES * 64;
constexpr uint32_t SMEM_BYTES = OFF_BAR + 512 + 1024;           // + alignment slack
constexpr uint32_t TMEM_COLS = 512;                             // S_0, S_1, O_0, O_1
constexpr uint64_t WAIT_CYCLES = 4000000000ull;                 // ~2 s
constexpr uint64_t DRAIN_CYCLES = 400000000ull;
constexpr float RESCALE_THRESHOLD = 8.f;  // O is rescaled when a row's maximum (base 2) grows by more
constexpr int E_TOP = 9;  // a query row's largest value, 16 keys' largest scale (or new value), is put at 2^9..2^10
constexpr float M_START = -1e30f;  // a reference before any key
// Exponents of queries, new keys and key scales are taken as they are where 2^(e -
// E_TOP) and its inverse are normal fp32 numbers; smaller ones count as E_MIN (what
// a row of queries below it loses, 2^-151 a value, is nothing beside keys of 7 *
// 2^100).  What a score is multiplied by, the row's factor times the keys', may
// underflow: it is at least FACTOR_MIN, and the row's at least ROW_MIN, as a
// factor of 0 would make NaN of masked scores, -infinity.  (Sums of products are
// below 2^30, so that such a score is 0 beside 1.)
constexpr int E_MIN = -117, E_MAX = 127;
constexpr float FACTOR_MIN = 0x1p-126f, ROW_MIN = 0x1p-149f, ROW_MAX = 0x1.fffffep127f;
// A unit's start and end in blocks of one tile (4 takes 183 us where 8 takes 161,
// 16 ragged trees of 64 nodes), and the least share worth a CTA: with 12 instead
// of 6 a tree of 32 nodes over 2000 keys takes 37 us instead of 31, one of 64 over
// 8192 43 instead of 41; with 4 they take 27 and 41, but 4 trees of 64 nodes over
// 300 keys 35 instead of 31.
constexpr int UNIT_COST = 8, LEAST = 6;

// Registers a thread by warpgroup (setmaxnreg), of the launch's 96.  The shares must add up to the launch's
// allocation, or the increase never returns; the host checks the compiled count.
constexpr int REGS_LAUNCH = 96, REGS_ISSUE = 80, REGS_NUMBERS = 80, REGS_SOFTMAX = 120;
static_assert(REGS_ISSUE + 2 * REGS_NUMBERS + 2 * REGS_SOFTMAX <= 5 * REGS_LAUNCH, "register split");

enum {
  B_KFULL = 0,   // [2] 8 arrivals
  B_VFULL = 2,   // [2] 8
  B_KEMPTY = 4,  // [2]
  B_VEMPTY = 6,  // [2]
  B_SFULL = 8,   // [2 tiles]
  B_PFULL = 10,  // [2 tiles] 4
  B_INFO = 12,   // [SLOTS] 2: a block's scales and keep bits
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
  Kv4Args a;
  int chunks;      // most units a (sequence, kv head)
  int split;       // 0: whole units, CTA by CTA
  int rows_cap;    // rows a piece's slot has room for
  int* list;       // [grid][8] cut units for k_kv4_join
  float* part_o;   // [grid][2][rows_cap][HD]
  float2* part_ml; // [grid][2][rows_cap]
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
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
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
// The eight products of a tile and a block (K = 16 each), one lane elected for
// all of them: descriptors differ in their low words, by constants; their high
// words are alike (1024 bytes between 8-row groups, version 1, 128-byte
// swizzle).  One statement, so that the operands move to uniform registers once.
constexpr uint32_t DESC_HI = (1024u >> 4) | (1u << 14) | (2u << 29);
// S[tmem d] = A . B^T, both from shared memory, K-major halves of 64 dims
__device__ __forceinline__ void mma_qk(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc) {
  asm volatile(
      "{\n\t.reg .pred z, o, e;\n\t.reg .b64 a, b;\n\t.reg .b32 t, h;\n\tmov.b32 h, %4;\n\t"
      "setp.ne.b32 z, 0, 0;\n\tsetp.eq.b32 o, 0, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
      "add.u32 t, %1, 0;\n\tmov.b64 a, {t, h};\n\tadd.u32 t, %2, 0;\n\tmov.b64 b, {t, h};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, z;\n\t"
      "add.u32 t, %1, 2;\n\tmov.b64 a, {t, h};\n\tadd.u32 t, %2, 2;\n\tmov.b64 b, {t, h};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, o;\n\t"
      "add.u32 t, %1, 4;\n\tmov.b64 a, {t, h};\n\tadd.u32 t, %2, 4;\n\tmov.b64 b, {t, h};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, o;\n\t"
      "add.u32 t, %1, 6;\n\tmov.b64 a, {t, h};\n\tadd.u32 t, %2, 6;\n\tmov.b64 b, {t, h};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, o;\n\t"
      "add.u32 t, %1, 1024;\n\tmov.b64 a, {t, h};\n\tadd.u32 t, %2, 1024;\n\tmov.b64 b, {t, h};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, o;\n\t"
      "add.u32 t, %1, 1026;\n\tmov.b64 a, {t, h};\n\tadd.u32 t, %2, 1026;\n\tmov.b64 b, {t, h};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, o;\n\t"
      "add.u32 t, %1, 1028;\n\tmov.b64 a, {t, h};\n\tadd.u32 t, %2, 1028;\n\tmov.b64 b, {t, h};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, o;\n\t"
      "add.u32 t, %1, 1030;\n\tmov.b64 a, {t, h};\n\tadd.u32 t, %2, 1030;\n\tmov.b64 b, {t, h};\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, o;\n\t"
      "}" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "n"(DESC_HI)
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
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
// 16 bytes of bf16 in dimension order to the tiles' order
__device__ __forceinline__ uint4 permute8(const uint4& v) {
  return make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410),
                    __byte_perm(v.y, v.w, 0x7632));
}
__device__ __forceinline__ float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // -126 <= e <= 127
__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Largest finite magnitude of a word's two bf16 values, packed like them.
__device__ __forceinline__ uint32_t top2(uint32_t top, uint32_t w) {
  const uint32_t mag = w & 0x7FFF7FFFu;
  return __vmaxu2(top, mag & ~__vcmpgeu2(mag, 0x7F807F80u));
}
// Exponent of a magnitude given as bf16 bits, in E_MIN..E_MAX.
__device__ __forceinline__ int expo_of(uint32_t bits) { return min(max((int)(bits >> 7) - 127, E_MIN), E_MAX); }
// 16 bytes of bf16 in the tiles' order times a power of two, as fp16
__device__ __forceinline__ uint4 to_f16(const uint4& v, float by) {
  auto two = [&](uint32_t w) { return pack_f16x2(lo_f(w) * by, hi_f(w) * by); };
  return make_uint4(two(v.x), two(v.y), two(v.z), two(v.w));
}
// 8 numbers (one word) times a scale, as fp16 in the tiles' order: 0x4C00 |
// (c << 6) is 16 + c; less24 is -24 times the scale
__device__ __forceinline__ uint4 scaled(uint32_t w, uint32_t s2, uint32_t less24) {
  auto two = [&](uint32_t v) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"((v & 0x03C003C0u) | 0x4C004C00u), "r"(s2), "r"(less24));
    return r;
  };
  return make_uint4(two(w << 6), two(w << 2), two(w >> 2), two(w >> 6));
}

// 8 numbers as bf16 in the tiles' order: 0x4300 | c is 128 + c
__device__ __forceinline__ uint4 numbers(uint32_t w) {
  auto two = [](uint32_t v) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"((v & 0x000F000Fu) | 0x43004300u), "r"(0x43084308u));
    return r;
  };
  return make_uint4(two(w), two(w >> 4), two(w >> 8), two(w >> 12));
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
  Kv4Cut cut;
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
    const Kv4Args& a = f.a;
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
  __device__ __forceinline__ int unit_cost(const Req& r) const { return UNIT_COST + r.blocks * r.w; }

  // every lane of a warp calls this
  __device__ __forceinline__ Walk(const ManyArgs& args) : f(args), cut(1, 1, 1) {
    const Kv4Args& a = f.a;
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
    cut = Kv4Cut(__reduce_add_sync(0xFFFFFFFFu, sum), gridDim.x, LEAST);
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
    const Kv4Args& a = f.a;
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
        const int from = max(0, cur - unit_base - UNIT_COST), to = min(cost, end - unit_base) - UNIT_COST;
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
  __device__ __forceinline__ int first_cta() const { return cut.share_of(unit_base + UNIT_COST); }
  __device__ __forceinline__ int last_cta() const {
    return cut.share_of(unit_base + UNIT_COST + (blocks - 1) * (two ? 2 : 1));
  }
  __device__ __forceinline__ int slot(int c) const { return 2 * c + (cut.start(c) < unit_base ? 1 : 0); }
};

__global__ void __launch_bounds__(THREADS, 1) k_kv4_attn_many(ManyArgs f) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ uint32_t s_tmem;
  __shared__ volatile int s_abort;
  const Kv4Args& a = f.a;
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
      if (i < B_KEMPTY || (i >= B_QE && i < B_QE + PIECES)) n = NUM_WARPS;
      if (i >= B_INFO && i < B_INFO + SLOTS) n = 2;
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
    // fp16 operands: format 0 where bf16 is 1 (bits 7..9, 10..12)
    constexpr uint32_t BF16 = (1u << 7) | (1u << 10);
    constexpr uint32_t IDESC_QK = idesc_bf16_f32(BM, BN, 0) & ~BF16, IDESC_PV = idesc_bf16_f32(BM, HD, 1);
    uint32_t nb = 0, np = 0, t_of[2] = {0, 0};  // blocks, pieces, steps of each tile so far
    bool ok = true;
    // descriptors' low words: a byte offset adds to them in units of 16
    const uint32_t q_lo = (uint32_t)smem_desc_sw128(sQ, 16, 1024), k_lo = (uint32_t)smem_desc_sw128(sK, 16, 1024);
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
      const int two = pc->two ? 1 : 0, steps = n << two;
      qt.next(two);
#pragma unroll 1
      for (int k = -2; k < steps; ++k) {
        const uint32_t x = k & 1;
        const uint32_t blk2 = nb + ((k + 2) >> two);
        if (two && !x && k + 2 < steps && !wait(B_KFULL + (blk2 & 1), blk2 >> 1)) break;
        if (k >= 0) {  // O_x (+)= P_x V
          const uint32_t blk = nb + (k >> two), st = blk & 1;
          if (!(two & x) && !wait(B_VFULL + st, blk >> 1)) break;  // tile 1: waited for by tile 0
          if (!wait(B_PFULL + x, t_of[x])) break;
          ++t_of[x];
          if (k == 0 && np > 0 && !wait(B_OFREE, np - 1)) break;
          tc_fence_after();
          mma_pv(tmem + 256 + x * 128, tmem + x * 128, v_lo + st * (TILE_BYTES >> 4), IDESC_PV, k >= 2);
          if (!two || x) {
            tc_commit(bar(B_VEMPTY + st));
            tc_commit(bar(B_SLOT + blk % SLOTS));
          }
        }
        if (k + 2 < steps) {  // S_x <- Q K^T
          const uint32_t blk = nb + ((k + 2) >> two), st = blk & 1;
          if (!two && !wait(B_KFULL + st, blk >> 1)) break;
          tc_fence_after();
          mma_qk(tmem + x * 128, q_lo + (two ? x : (uint32_t)qt.tile) * (TILE_BYTES >> 4), k_lo + st * (TILE_BYTES >> 4), IDESC_QK);
          tc_commit(bar(B_SFULL + x));
          if (!two || x) tc_commit(bar(B_KEMPTY + st));
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
    } else {
      // ---------------- keys' scales, ahead of their rows ----------------
      // Thread i: keys 2i, 2i + 1 of a block, in run i / 8 of its eight.
      const int i = tid - 64, run_i = i >> 3;
      const uint32_t per_page = (uint32_t)a.Hkv << (a.shift - 4), in_page = (1u << (a.shift - 4)) - 1u;
      uint32_t nb = 0;
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
        uint32_t run = 0, kw = 0, vw = 0;
        bool in = false;
        auto fetch = [&](int blk) {
          in = (unsigned)id < (unsigned)a.n_pages;
          run = in ? id * per_page + ((uint32_t)pc.gh << (a.shift - 4)) + (((uint32_t)blk * (BN / 16) + run_i) & in_page) : 0u;
          kw = reinterpret_cast<const uint32_t*>(a.ks)[(uint64_t)run * 8u + (i & 7)];
          vw = reinterpret_cast<const uint32_t*>(a.vs)[(uint64_t)run * 8u + (i & 7)];
          // the rows of its run: a line of K and one of V, asked into L2
          prefetch_l2(a.kc + (uint64_t)run * 1024u + (i & 7) * 128);
          prefetch_l2(a.vc + (uint64_t)run * 1024u + (i & 7) * 128);
        };
        if (pc.s0 < to) fetch(pc.s0);
        for (int blk = pc.s0; blk < s1; ++blk, ++nb) {
          const int slot = nb % SLOTS;
          const bool fresh = blk >= pc.cached;
          const uint32_t run_now = run;
          int left;  // keys of the run that count
          uint32_t top, k0 = 0, k1 = 0, v2 = 0x3F803F80u;
          if (!fresh) {
            const long long more = pc.kvl - ((long long)blk * BN + 16 * run_i);
            left = in ? (int)min(16ll, max(0ll, more)) : 0;
            if (!in && more > 0 && (i & 7) == 0) fc_flag(FC_ERR_WORD(a.err), FC_EBIT_INVALID);
            // a key that does not count: whatever stands there
            const uint32_t some = 2 * (i & 7) + 1 < left ? 0xFFFFFFFFu : (2 * (i & 7) < left ? 0xFFFFu : 0u);
            k0 = kw & some;
            v2 = vw & some;
            top = top2(0u, k0);
            k1 = k0 >> 16;
            k0 &= 0xFFFFu;
            if (blk + 1 < to) {
              id = id_next;
              fetch(blk + 1);
              id_next = look_up(blk + 2);
            }
          } else {
            left = a.k_new ? min(16, max(0, pc.nn - 16 * run_i)) : 0;
            const uint4* src = reinterpret_cast<const uint4*>(a.k_new + (((size_t)pc.b * a.Hkv + pc.gh) * a.n_pad + 16 * run_i) * HD);
            top = 0;
#pragma unroll 8
            for (int e = i & 7; e < left * (HD / 8); e += 8) {
              const uint4 k = src[e];
              top = top2(top2(top2(top2(top, k.x), k.y), k.z), k.w);
            }
          }
          top = max(top & 0xFFFFu, top >> 16);
#pragma unroll
          for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
          const int ek = expo_of(top);
          const float by = pow2i(E_TOP - ek);
          if (nb >= SLOTS && !(ok = warp_wait(bar(B_SLOT + slot), (nb / SLOTS - 1) & 1, &s_abort))) break;
          if ((i & 7) == 0) {
            reinterpret_cast<uint16_t*>(smem + OFF_KEEP + slot * 16)[run_i] = (uint16_t)((1u << left) - 1u);
            reinterpret_cast<float*>(smem + OFF_BACK)[slot * (BN / 16) + run_i] = pow2i(ek - E_TOP);
            reinterpret_cast<uint32_t*>(smem + OFF_RUN)[slot * (BN / 16) + run_i] = fresh ? __float_as_uint(by) : run_now;
          }
          reinterpret_cast<float2*>(smem + OFF_VS)[slot * (BN / 2) + i] = make_float2(lo_f(v2), hi_f(v2));
          const float f0 = lo_f(k0) * by, f1 = lo_f(k1) * by;
          reinterpret_cast<uint4*>(smem + OFF_KS)[slot * (BN / 2) + i] =
              make_uint4(pack_f16x2(f0, f0), pack_f16x2(-24.f * f0, -24.f * f0), pack_f16x2(f1, f1),
                         pack_f16x2(-24.f * f1, -24.f * f1));
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(B_INFO + slot));
        }
      }
    }
  } else if (warp >= 12) {
    // ---------------- numbers to tiles ----------------
    // Warp w has rows 16w .. 16w + 15 of a block, one run of a page: lane (rho,
    // c) rows rho and rho + 8, 16 bytes c of their 64.  Eight lanes in turn have
    // four rows of one 64-dim half, so that their stores fall in different banks.
    const int w = warp - 12, c = (lane & 1) | ((lane >> 4) << 1), rho = (lane >> 1) & 7;
    uint32_t dst[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      dst[i] = (c >> 1) * HALF_BYTES + (16 * w + rho) * 128 + ((((c & 1) * 4 + i) ^ rho) << 4);
    Piece pc = {};
    uint4 kr[2], vr[2];
    uint32_t nb = 0;
    bool ok = true;
    auto info = [&](uint32_t blk) {
      return warp_wait(bar(B_INFO + blk % SLOTS), (blk / SLOTS) & 1, &s_abort);
    };
    const uint32_t* runs = reinterpret_cast<const uint32_t*>(smem + OFF_RUN) + w;
    auto fetch = [&](const uint8_t* codes, uint32_t run, uint4 (&x)[2]) {
      const uint4* src = reinterpret_cast<const uint4*>(codes + (uint64_t)run * 1024u) + rho * 4 + c;
      x[0] = src[0];
      x[1] = src[32];
    };
    const size_t no_row = ~(size_t)0;
    auto new_row = [&](int j) {
      return a.k_new && j < pc.nn ? (((size_t)pc.b * a.Hkv + pc.gh) * a.n_pad + j) * HD : no_row;
    };
    // The piece's queries: a row 16 lanes, 16 rows at a time, times a power of two.
    auto stage_q = [&](uint32_t np, int tile) {
      float* back = reinterpret_cast<float*>(smem + OFF_QE) + np % PIECES * ROWS;
      const int ch = lane & 15, passes = (pc.two ? 2 : 1) * BM / 16;
#pragma unroll 1
      for (int p0 = 0; p0 < passes; p0 += 2) {
        uint4 v[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int r = 16 * (p0 + k) + 2 * w + (lane >> 4);
          v[k] = make_uint4(0, 0, 0, 0);
          if (r < pc.rows) {
            const int rr = pc.row0 + r, i = rr / a.G, hh = rr - i * a.G;
            v[k] = reinterpret_cast<const uint4*>(a.q + (((size_t)pc.b * a.n_pad + i) * a.H + pc.gh * a.G + hh) * HD)[ch];
          }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int r = 16 * (p0 + k) + 2 * w + (lane >> 4);
          const uint32_t sign = 0x7FFF7FFFu;
          uint32_t top = __vmaxu2(__vmaxu2(v[k].x & sign, v[k].y & sign), __vmaxu2(v[k].z & sign, v[k].w & sign));
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) top = __vmaxu2(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
          const int ex = expo_of(max(top & 0xFFFFu, top >> 16));
          if (ch == 0) back[r] = pow2i(ex - E_TOP);
          *reinterpret_cast<uint4*>(smem + OFF_Q + (tile + (r >> 7)) * TILE_BYTES + (ch >> 3) * HALF_BYTES + (r & 127) * 128 +
                                    (((ch & 7) ^ (r & 7)) << 4)) = to_f16(permute8(v[k]), pow2i(E_TOP - ex));
        }
      }
    };
    auto store = [&](uint32_t tile, const uint4 (&x)[2], auto&& convert) {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        unsigned char* t = smem + tile + p * 1024;
        *reinterpret_cast<uint4*>(t + dst[0]) = convert(p, x[p].x);
        *reinterpret_cast<uint4*>(t + dst[1]) = convert(p, x[p].y);
        *reinterpret_cast<uint4*>(t + dst[2]) = convert(p, x[p].z);
        *reinterpret_cast<uint4*>(t + dst[3]) = convert(p, x[p].w);
      }
    };
    auto store_new = [&](uint32_t tile, const __nv_bfloat16* src, auto&& convert) {  // the new rows, zeros past them
#pragma unroll 2
      for (int e = lane; e < 256; e += 32) {
        const int j = 16 * w + (e >> 4), ch = e & 15;
        const size_t row = new_row(j);
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row != no_row) v = convert(permute8(reinterpret_cast<const uint4*>(src + row)[ch]), e >> 4);
        *reinterpret_cast<uint4*>(smem + tile + (ch >> 3) * HALF_BYTES + j * 128 + (((ch & 7) ^ (j & 7)) << 4)) = v;
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
        fetch(a.kc, run, kr);
        fetch(a.vc, run, vr);
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
        if (nb >= 2 && !(ok = warp_wait(bar(B_KEMPTY + st), ((nb >> 1) - 1) & 1, &s_abort))) break;
        const uint2* ks = reinterpret_cast<const uint2*>(smem + OFF_KS) + slot * BN + 16 * w + rho;
        const uint2 s[2] = {ks[0], ks[8]};
        store(OFF_K + st * TILE_BYTES, kr, [&](int p, uint32_t v) { return scaled(v, s[p].x, s[p].y); });
        done(B_KFULL + st);
        if (more) {
          if (!(ok = info(nb + 1))) break;
          run = runs[(nb + 1) % SLOTS * (BN / 16)];
          fetch(a.kc, run, kr);
        }
        if (nb >= 2 && !(ok = warp_wait(bar(B_VEMPTY + st), ((nb >> 1) - 1) & 1, &s_abort))) break;
        store(OFF_V + st * TILE_BYTES, vr, [](int, uint32_t v) { return numbers(v); });
        done(B_VFULL + st);
        if (more) fetch(a.vc, run, vr);
      }
      if (ok && to < s1) {  // the new tokens' block
        const int st = nb & 1;
        if (!(ok = info(nb))) break;
        if (nb >= 2 && !(ok = warp_wait(bar(B_KEMPTY + st), ((nb >> 1) - 1) & 1, &s_abort))) break;
        const float by = __uint_as_float(runs[nb % SLOTS * (BN / 16)]);
        store_new(OFF_K + st * TILE_BYTES, a.k_new, [&](const uint4& v, int) { return to_f16(v, by); });
        done(B_KFULL + st);
        if (nb >= 2 && !(ok = warp_wait(bar(B_VEMPTY + st), ((nb >> 1) - 1) & 1, &s_abort))) break;
        // A value that is not finite becomes 0, as no weight of 0 would take it
        // out of the rows that do not see its token; those that do are NaN.
        uint32_t bad = 0;
        store_new(OFF_V + st * TILE_BYTES, a.v_new, [&](const uint4& v, int j) {
          auto finite = [&](uint32_t x) {
            const uint32_t not_finite = __vcmpgeu2(x & 0x7FFF7FFFu, 0x7F807F80u);
            if (not_finite) bad |= 1u << j;
            return x & ~not_finite;
          };
          return make_uint4(finite(v.x), finite(v.y), finite(v.z), finite(v.w));
        });
        bad = __reduce_or_sync(0xFFFFFFFFu, bad);
        if (lane == 0) reinterpret_cast<uint16_t*>(smem + OFF_BAD)[np % PIECES * NUM_WARPS + w] = (uint16_t)bad;
        done(B_VFULL + st);
        ++nb;
      }
    }
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
      const int lr = row_of(pc), i = (pc->row0 + lr) / a.G;
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
          fminf(fmaxf(a.scale_log2 * reinterpret_cast<const float*>(smem + OFF_QE)[np % PIECES * ROWS + row_of(pc)], ROW_MIN), ROW_MAX);
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
        if (!(ok = warp_wait(bar(B_SFULL + x), t & 1, &s_abort))) break;
        tc_fence_after();
        if (__builtin_expect(masked, 0)) {  // masked scores are overwritten by -inf
          uint64_t sees[2] = {~0ull, ~0ull};
          if (j >= n_cached) seen(pc, sees);
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
        // The row's scores come 32 at a time, once for the maximum, once for P:
        // one short loop each, as two bodies with loads in flight beside them
        // took longer (1160 us where this takes 1100): the roles share the
        // instruction cache and the other warps cover the loads.
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
        const ulonglong2* vs4 = reinterpret_cast<const ulonglong2*>(smem + OFF_VS + slot * BN * 4);
        auto weigh = [&](int q, const uint32_t (&sv)[32]) {  // over scores already read
          uint32_t pk[16];
          const float2 bk = back[q];
#pragma unroll
          for (int g = 0; g < 8; ++g) {  // 4 keys, their value scales in one load
            const ulonglong2 v4 = vs4[q * 8 + g];
            const float cz = fmaxf(c_row * (g < 4 ? bk.x : bk.y), FACTOR_MIN);
            const uint64_t c2 = f2_pack(cz, cz);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const int k = 4 * g + 2 * u;
              float p0, p1;
              f2_unpack(f2_fma(f2_pack(__uint_as_float(sv[k]), __uint_as_float(sv[k + 1])), c2, neg), p0, p1);
              const uint64_t pp = f2_pack(exp2_fast(p0), exp2_fast(p1));
              sum[u] = f2_add(sum[u], pp);
              f2_unpack(f2_mul(pp, u ? v4.y : v4.x), p0, p1);
              pk[2 * g + u] = pack_bf16x2(p0, p1);
            }
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
      const int lr = row_of(pc), rr = pc->row0 + lr, i = rr / a.G, hh = rr - i * a.G;
      const bool row_ok = lr < pc->rows;
      __nv_bfloat16* dst = a.out + (((size_t)pc->b * a.n_pad + (row_ok ? i : 0)) * a.H + pc->gh * a.G + hh) * HD;
      const size_t slot = (size_t)pc->slot * f.rows_cap + lr;
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
#pragma unroll 1
      for (int cc = two ? 0 : 4 * x; cc < (two ? 8 : 4 * x + 4); ++cc) {
        uint32_t o[16];
        float v[16];
        tmem_ld16(tO0 + cc * 16, o);
        tc_wait_ld();
#pragma unroll
        for (int u = 0; u < 16; ++u) v[u] = __uint_as_float(o[u]) * k0;
        if (both) {
          tmem_ld16(tO0 + 128 + cc * 16, o);
          tc_wait_ld();
#pragma unroll
          for (int u = 0; u < 16; ++u) v[u] = fmaf(__uint_as_float(o[u]), k1, v[u]);
        }
        if (row_ok) {
#pragma unroll
          for (int u = 0; u < 16; u += 8) {  // out of the tiles' order: 0 4 1 5 2 6 3 7
            if (whole) {
              *reinterpret_cast<uint4*>(dst + cc * 16 + u) =
                  make_uint4(pack_bf16x2(v[u], v[u + 2]), pack_bf16x2(v[u + 4], v[u + 6]),
                             pack_bf16x2(v[u + 1], v[u + 3]), pack_bf16x2(v[u + 5], v[u + 7]));
            } else {
              float4* po = reinterpret_cast<float4*>(f.part_o + slot * HD + cc * 16 + u);
              po[0] = make_float4(v[u], v[u + 2], v[u + 4], v[u + 6]);
              po[1] = make_float4(v[u + 1], v[u + 3], v[u + 5], v[u + 7]);
            }
          }
        }
      }
      if (!whole && row_ok && (two || x == 0)) f.part_ml[slot] = make_float2(m_all, l);
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
// second piece CTA c of k_kv4_attn_many began with, 8 of its rows, a warp each.
__global__ void __launch_bounds__(256) k_kv4_join(ManyArgs f) {
  const Kv4Args& a = f.a;
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
  const int i = (row0 + r) / a.G, hh = (row0 + r) - i * a.G;
  __nv_bfloat16* dst = a.out + (((size_t)b * a.n_pad + i) * a.H + gh * a.G + hh) * HD + 4 * lane;
  *reinterpret_cast<uint2*>(dst) =
      make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
}

int rows_of_chunk(int n_pad, int G) { return std::min(ROWS, n_pad * G); }

size_t list_bytes(int grid) { return ((size_t)grid * 32 + 255) / 256 * 256; }
size_t slot_bytes(int rows) { return (size_t)rows * (HD * sizeof(float) + sizeof(float2)); }

constexpr int FULL_GRID = 152;

}  // namespace

size_t kv4_attn_many_workspace(int batch, int n_pad, int H, int Hkv) {
  (void)batch;
  return KV4_WS_COUNTERS + list_bytes(FULL_GRID) + (size_t)FULL_GRID * 2 * slot_bytes(rows_of_chunk(n_pad, H / Hkv));
}

fc_status kv4_attn_many(const Kv4Args& a, void* ws, size_t ws_bytes, cudaStream_t s) {
  static std::atomic<unsigned long long> done{0};
  const fc_status st = fc_once_per_device(done, [](int) {
    cudaFuncAttributes attr;
    if (cudaFuncGetAttributes(&attr, k_kv4_attn_many) != cudaSuccess) return FC_ERR_CUDA;
    if (attr.numRegs < REGS_LAUNCH) return FC_ERR_INTERNAL;  // the register split would not add up
    return fc_cuda_status(cudaFuncSetAttribute(k_kv4_attn_many, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES));
  });
  if (st != FC_OK) return st;
  ManyArgs f{a, 0, 1, rows_of_chunk(a.n_pad, a.G), nullptr, nullptr, nullptr};
  f.chunks = (a.n_pad * a.G + ROWS - 1) / ROWS;
  const long long units = (long long)a.B * a.Hkv * f.chunks;
  if (units > 0x7FFFFFFFll) return FC_ERR_UNSUPPORTED;
  const long long longest = (((long long)a.max_pages << a.shift) + BN - 1) / BN + 1;
  const bool fits = units * (UNIT_COST + 2 * longest) <= 0x7FFFFFFFll;
  int grid = (int)std::min<long long>(FULL_GRID, units * ((UNIT_COST + 2 * longest) / LEAST));
  auto need = [&] { return KV4_WS_COUNTERS + list_bytes(grid) + (size_t)grid * 2 * slot_bytes(f.rows_cap); };
  while (grid > 1 && ws && need() > ws_bytes) --grid;
  // a workspace for fewer CTAs than whole units would fill: whole units (16
  // trees of 32 nodes over 2000 keys on two CTAs 1.91 ms, whole units 0.04)
  if (!ws || !fits || need() > ws_bytes || grid < std::min<long long>(FULL_GRID, units)) {
    f.split = 0;
    grid = (int)std::min<long long>(units, FULL_GRID);
  } else {
    unsigned char* p = static_cast<unsigned char*>(ws) + KV4_WS_COUNTERS;
    f.list = reinterpret_cast<int*>(p);
    f.part_o = reinterpret_cast<float*>(p + list_bytes(grid));
    f.part_ml = reinterpret_cast<float2*>(f.part_o + (size_t)grid * 2 * f.rows_cap * HD);
  }
  k_kv4_attn_many<<<grid, THREADS, SMEM_BYTES, s>>>(f);
  if (f.split && grid > 1) k_kv4_join<<<dim3(grid, (f.rows_cap + 7) / 8), 256, 0, s>>>(f);
  return FC_CHECK_LAUNCH();
}
