// Attention of many new tokens per sequence, on the 5th-generation tensor cores: whole prompts over their own packed keys and
// values, and chunks of new tokens over the paged cache (E4M3, bf16 or 4-bit codes).  Causal, with a window or without,
// sink logit per query head (paper, Sections "Window attention for long-context inference" and "Optimized Scenarios").
//
//     s_j = sm_scale k_scale (q . k_j),  M = max(max_j s_j, sink),  Z = e^(sink - M) + sum_j e^(s_j - M),
//     out = v_scale sum_j e^(s_j - M) v_j / Z,    j over the keys [p + 1 - W, p] of the token at position p
//
// in one pass over the keys with a running maximum and sum.  A tile of rows is 16 tokens x the 8 query heads of one KV head
// (128 rows, so that one tile of keys serves all of them and a window wastes at most 16 tokens of it), a tile of keys 128.
//
//  * Four streams, each with a warpgroup for the softmax (thread = row) and a warp that issues its MMAs.  A stream computes
//    S = Q K^T (128 rows x 64 keys: half a tile) into 64 columns of tensor memory, its threads read their rows, write the weights
//    P over them as the A operand of O += P V, and O stays in 64 columns of its own: 4 x (64 + 64) = all 512 columns.  Streams
//    share nothing until their rows are done; then they join through tensor memory, each for a part of the channels.  The two
//    halves of a tile are two streams, not one of twice the width, so that every scheduler has four softmax warps: the special
//    function unit (16 exponentials a clock and SM), the busiest unit at 64 %, is fed while others wait for loads and products.
//    What bounds a long prompt is that each stream is a chain (S, exponentials, P V, next S) and four do not cover each other's waits.
//    Measured on a prompt of 8192 tokens when it was chosen: 740 us; two streams of 128 keys, with S and P apart so that the next S is
//    computed early, 966; the same with two threads to a row 802.  Now 600 to 610 (900 TFLOP/s).
//  * A group of 64, 32 or 16 tokens is 4, 2 or 1 tiles of rows with 1, 2 or 4 streams each; these take the halves of the tiles of keys
//    in turn and join at the end.  Large groups fetch (and convert) a tile of keys once for many rows and have nothing to join, small
//    ones make more items of few tokens.
//  * One warp plans the work and loads packed keys and values by TMA, one loads queries, one looks at the values of tiles that not
//    every row sees (below).  Over a code cache one copies blocks through the block table, and four convert them: K to bf16, V to f16,
//    both exact for E4M3 and for E2M1 times its scale.  Over a bf16 cache these four copy to where the MMAs read.
//  * The reference that weights are relative to is the largest logit of a row's first 32 keys that it sees any of.  It is looked at
//    again, and O rescaled, only where the weights sum to more than the type of P can take: usual tiles need no maximum.  The weights
//    of a bf16 V are bf16 (half a step, 2^-8 of each, the rounding of the output itself) with float32's range: the limit is 2^40.
//    Those of a converted V are f16 (2^-11) and lie at 2^9 of their value, so that the sum of 64 at the reference stays below the
//    limit, f16's largest number, and weights down to 2^-23 of the reference keep all their bits.  A reference is raised by whole
//    powers of two, so that the weights of the keys before, in f16 already, are scaled exactly; it then lies less than a factor of two
//    above the largest.  Sums are float32.
//  * A quarter of the exponentials of usual tiles goes through a polynomial on the FMA units.  The special function unit's queue is
//    shared with shared and tensor memory: a warp that fills it holds up the loads and arrivals of the others (8192 tokens: none of
//    them 775 us, an eighth 670, a quarter 643, a third 641, half 736).
//  * Tiles at an edge (diagonal, window, first of a row) go 32 keys at a time through code of half the length: with few tiles per row
//    every warp fetches its instructions anew (prompts with a window of 128: 64 at a time 280 us, 32 at a time 252).
//  * Work comes by request (cluster launch control): a CTA asks for the next block of the grid while it works on one.  Blocks are
//    ordered long ones first within a sequence.
//  * MMAs and copies are issued by one elected lane out of a converged warp, with operands that the compiler knows to be uniform
//    (broadcast by a shuffle): otherwise every MMA costs 75 to 150 clocks to issue, which alone took 200 us of 950.
//  * 0 x NaN: a tile of V that some row of the group does not see is searched for infinities and NaN before its product.  They
//    are replaced by zero, and the rows that do see them get them added at the end, read again from where they come from.
//
// Every wait is bounded: one that runs out sets PUZZLE_DEV_WAIT_EXPIRED and a flag upon which every role leaves its loop.  When all have,
// those that set something going (products, copies, the request for work) wait for it, again with a limit, so that none is in
// flight when shared and tensor memory are given back.  Copies that no barrier of the others follows are waited for in any case.
#include <cuda_fp16.h>

#include <algorithm>

#include "kv_fp4.cuh"
#include "prompt_attn.cuh"

namespace puzzle {
namespace {

constexpr int kRowTokens = 16;              // tokens of a tile of rows
constexpr int TK = 128;                     // keys of a tile
constexpr int NBLK = TK / kBlock;
constexpr int kTileBytes = TK * kHeadDim * 2;
constexpr int kRing = 4;                    // work records: of the item being worked on and the next ones
constexpr int kShortTiles = 4;              // items of no more tiles are asked for that far ahead, longer ones one ahead
constexpr unsigned kFull = 0xffffffffu;
constexpr float kPoly5 = 0.0013274633f, kPoly4 = 0.0096719619f, kPoly3 = 0.0555067845f, kPoly2 = 0.2402223498f,
                kPoly1 = 0.6931470633f;
constexpr float kUnset = -3.402823466e38f;  // a reference that no logit is below
constexpr float kLarge = 1048576.f;         // references beyond 2^20: see there
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kHalf = NBLK / 2;             // blocks of a stream's half of a tile
// tensor memory: S (and P over it) of the four streams, then O
constexpr int kTmemS = 0, kTmemO = 256;

// ROWS: tiles of rows that a group can have (4: any group; 1: of 16 tokens alone, which leaves room for more tiles of keys).
template <int SRC, int ROWS>
struct Cfg {
  static constexpr bool kPaged = SRC != kSrcPacked;
  static constexpr bool kCodes = SRC == kSrcFp8 || SRC == kSrcFp4;
  static constexpr int kThreads = kPaged ? 896 : 768;
  static constexpr int kStages = kCodes ? (ROWS == 1 ? 4 : 3) : (ROWS == 1 ? 6 : 4);             // tiles of K and V in the form the MMAs read
  static constexpr int kBlockBytes = SRC == kSrcFp8 ? kBlock * kHeadDim : (SRC == kSrcFp4 ? kFp4BlockBytes : 0);
  static constexpr int kCodeTile = 2 * NBLK * kBlockBytes;   // codes of K and V of a tile as they lie in the cache
  // tiles whose copies are in flight; a bf16 tile is copied to where the MMAs read it, and has to leave one of these places
  static constexpr int kCopySlots = SRC == kSrcFp8 ? (ROWS == 1 ? 4 : 3) : (SRC == kSrcFp4 ? (ROWS == 1 ? 6 : 5) : (ROWS == 1 ? 4 : 3));
  static constexpr int kCodeStages = kCodes ? kCopySlots : 0;
  static constexpr int kFullArrivals = kPaged ? 4 : 1;
  // Register shares of the softmax warpgroups and of the others.  They come out of what the launch has: 65536 / threads rounded
  // down to 8 each, 72 x 896 and 80 x 768.
  static constexpr int kRegsSoftmax = 96, kRegsOther = kPaged ? 40 : 48;
  static_assert(512 * kRegsSoftmax + (kThreads - 512) * kRegsOther <= kThreads * (65536 / kThreads / 8 * 8), "more than there are");
  static constexpr float kShift = kCodes ? 9.f : 0.f;                  // weights lie at 2^shift of their value
  static constexpr float kMuch = kCodes ? 65000.f : 1.0995116e12f;     // sum of 64 weights that calls for another reference
  static constexpr int kSmem = ROWS * kTileBytes + 2 * kStages * kTileBytes + kCodeStages * kCodeTile;
};

struct Record {
  int on, b, kvh, row0, ntok, pos0, kb0, kb_end, part, bad_v;
};
struct Ctl {
  uint64_t rec_full[kRing], rec_empty[kRing];
  uint64_t q_full[4], q_empty[4];                         // of the tiles of rows
  uint64_t k_full[6], k_empty[6], v_full[6], v_empty[6], v_ok[6];
  uint64_t s_full[4], p_full[4], o_full[4], o_empty[4];   // of the streams
  uint64_t join_full[4];
  uint64_t ended[4];                                      // all products of a stream
  uint64_t next_full;
  alignas(16) uint4 next;   // answer to a request for work
  uint64_t copied[4][8];         // of a warp's blocks; of a tile's codes: the first row
  uint64_t codes_empty[8];
  Record rec[kRing];
  int asked, loaded, q_loaded[4];   // at the end of the warps that did it: requests for work, tiles, tiles of queries
  float2 join[2][4][128];   // by turns: reference and sum of a stream's rows
  uint32_t tmem;
  volatile int abort;
};

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Matrix descriptor of a tile with 128-byte rows and the 128-byte swizzle, eight rows every 1024 bytes.  `lo`: its address in units
// of 16 bytes, plus kDescLo.
constexpr uint32_t kDescLo = 1u << 16, kDescHi = 64u | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint64_t desc128(uint32_t lo) { return (uint64_t)kDescHi << 32 | lo; }
__device__ __forceinline__ void umma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
#define PZ_R32(r, b) \
  "=r"(r[b + 0]), "=r"(r[b + 1]), "=r"(r[b + 2]), "=r"(r[b + 3]), "=r"(r[b + 4]), "=r"(r[b + 5]), "=r"(r[b + 6]), \
      "=r"(r[b + 7]), "=r"(r[b + 8]), "=r"(r[b + 9]), "=r"(r[b + 10]), "=r"(r[b + 11]), "=r"(r[b + 12]), "=r"(r[b + 13]), \
      "=r"(r[b + 14]), "=r"(r[b + 15]), "=r"(r[b + 16]), "=r"(r[b + 17]), "=r"(r[b + 18]), "=r"(r[b + 19]), "=r"(r[b + 20]), \
      "=r"(r[b + 21]), "=r"(r[b + 22]), "=r"(r[b + 23]), "=r"(r[b + 24]), "=r"(r[b + 25]), "=r"(r[b + 26]), "=r"(r[b + 27]), \
      "=r"(r[b + 28]), "=r"(r[b + 29]), "=r"(r[b + 30]), "=r"(r[b + 31])
#define PZ_V32(r) \
  "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), \
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), \
      "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), \
      "r"(r[31])
// 32 columns of the warp's 32 lanes.
#define PZ_LIST32 \
  "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}"
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 " PZ_LIST32 ", [%32];" : PZ_R32(r, 0) : "r"(taddr));
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], " PZ_LIST32 ";" ::PZ_V32(r), "r"(taddr) : "memory");
}

#define PZ_LIST16 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}"
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 " PZ_LIST16 ", [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                 "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], " PZ_LIST16 ";" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
               "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
               "r"(r[14]), "r"(r[15]), "r"(taddr)
               : "memory");
}

// Pairs of floats, one instruction for both.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// 2^x for two arguments on the FMA units: x = i + f with i the nearest integer, 2^f by a polynomial of degree five with constant 1,
// fitted to the relative error on [-1/2, 1/2] (1.11e-7 at most, 1.55e-7 with float32's roundings), i added to the exponent.  Arguments
// below -125 give 2^-125; those above 126, and NaN, nothing of use.
__device__ __forceinline__ void exp2_poly(uint64_t x2, float& e0, float& e1) {
  float x0, x1;
  unpack2(x2, x0, x1);
  x2 = pack2(fmaxf(x0, -125.f), fmaxf(x1, -125.f));
  const uint64_t magic = pack2(12582912.f, 12582912.f), unmagic = pack2(-12582912.f, -12582912.f), minus = pack2(-1.f, -1.f);
  const uint64_t t = add2(x2, magic);                        // its low bits hold i
  const uint64_t f = fma2(add2(t, unmagic), minus, x2);
  uint64_t p = pack2(kPoly5, kPoly5);
  p = fma2(p, f, pack2(kPoly4, kPoly4));
  p = fma2(p, f, pack2(kPoly3, kPoly3));
  p = fma2(p, f, pack2(kPoly2, kPoly2));
  p = fma2(p, f, pack2(kPoly1, kPoly1));
  p = fma2(p, f, pack2(1.f, 1.f));
  float t0, t1, p0, p1;
  unpack2(t, t0, t1);
  unpack2(p, p0, p1);
  e0 = __int_as_float(__float_as_int(p0) + (__float_as_int(t0) << 23));
  e1 = __int_as_float(__float_as_int(p1) + (__float_as_int(t1) << 23));
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, int c0, int c1, int c2, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
      : "memory");
}
// 16 bytes from global to shared memory, zeros if !on.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
// `bytes` bytes (a multiple of 16) from global to shared memory, counted on an mbarrier.
__device__ __forceinline__ void bulk_copy(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
               "r"(bar)
               : "memory");
}
// One arrival of this thread once its copies so far have landed (the barrier's count includes it).
__device__ __forceinline__ void cp_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cp_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// All threads of the CTA, from either side of the split of registers (code behind the join has to do with the smaller share).
__device__ __forceinline__ void sync_cta() { asm volatile("barrier.sync 0;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void regs_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
__device__ __forceinline__ void st_shared16(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
// Two f16 values, both exact in bf16.
__device__ __forceinline__ uint32_t f16x2_to_bf16x2(uint32_t h) { return f32x2_to_bf16x2(f16_lo_to_f32(h), f16_hi_to_f32(h)); }

// The lowest n of 32 bits.
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : (n >= 32 ? 0xffffffffu : (1u << n) - 1u); }

// The 16 columns of weights that a thread has written, times alpha (a power of two).
template <bool F16>
__device__ __forceinline__ void rescale_weights(uint32_t at, float alpha) {
  uint32_t y[16];
  tmem_wait_st();
  tmem_ld16(at, y);
  tmem_wait_ld();
  const uint32_t a = f32x2_to_bf16x2(alpha, alpha);
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    if constexpr (F16) y[j] = f32x2_to_f16x2(f16_lo_to_f32(y[j]) * alpha, f16_hi_to_f32(y[j]) * alpha);   // alpha may be below f16
    else asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(y[j]) : "r"(a));
  }
  tmem_st16(at, y);
}

// Work by request: a CTA asks for a block of the grid that has not been started, and works in its place.  The answer goes to 16
// bytes of shared memory.
__device__ __forceinline__ void request_block(uint32_t dst, uint32_t bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(dst), "r"(bar)
               : "memory");
}
// The block's index, -1: there is none left.
__device__ __forceinline__ int granted_block(uint32_t src) {
  uint32_t ok, x;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b128 a;\n\t"
      "ld.shared.b128 a, [%2];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n\t"
      "selp.u32 %0, 1, 0, p;\n\tmov.u32 %1, 0;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, a;\n\t}"
      : "=r"(ok), "=r"(x)
      : "r"(src)
      : "memory");
  return ok ? (int)x : -1;
}

// Has the phase with this parity completed?
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}

// Waits by whole warps: one decision for the 32 lanes.
struct Waiter {
  Ctl* C;
  int32_t* status;
  __device__ __forceinline__ bool operator()(const uint64_t& bar, uint32_t parity) const {
    const uint32_t a = smem_u32(&bar);
    bool ok = mbar_try_wait(a, parity);
    if (__all_sync(kFull, ok)) return true;
    return slow(a, parity);
  }
  __device__ __forceinline__ bool slow(uint32_t a, uint32_t parity) const {
    bool ok = false;
    for (uint32_t i = 0; i < (1u << 24); ++i) {   // some waits last as long as an item does: more than a second, 10^7 keys and more
      if (mbar_try_wait(a, parity)) { ok = true; break; }
      if (C->abort) break;
      if (i > 64) __nanosleep(64);
    }
    ok = __all_sync(kFull, ok);
    if (!ok && !C->abort) {
      if (status) atomicOr(status, (int)PUZZLE_DEV_WAIT_EXPIRED);
      C->abort = 1;
    }
    return ok;
  }
};

// What stream st does of a record, `turns` streams to a tile of rows: its tokens, and of the half tiles [j_lo, j_hi) that they see
// those from j0 on, every turns-th.
struct Share {
  int pos, ntok, j_lo, j_hi, j0, turns, end;
  __device__ __forceinline__ Share(const Record& r, int st, int turns_, int window) : turns(turns_) {
    const int first = kRowTokens * (st / turns);
    pos = r.pos0 + first;
    ntok = min(max(r.ntok - first, 0), kRowTokens);
    const int hi = pos + ntok;                                              // behind the last key that one of them sees
    const int lo = window > 0 ? max(pos - window + 1, 0) : 0;
    end = ntok > 0 ? min(r.kb_end, hi > 0 ? (hi + kBlock - 1) / kBlock : 0) - r.kb0 : 0;   // blocks
    j_lo = max(lo / kBlock - r.kb0, 0) / kHalf;
    j_hi = end > 0 ? (end + kHalf - 1) / kHalf : 0;
    j0 = j_lo + ((st - j_lo) & (turns - 1));
  }
  __device__ __forceinline__ bool any() const { return j_hi > j_lo; }      // one of the streams of these tokens
  __device__ __forceinline__ bool on() const { return j_hi > j0; }
  __device__ __forceinline__ bool last(int j) const { return j + turns >= j_hi; }
  __device__ __forceinline__ int blocks(int j) const { return min(end - j * kHalf, kHalf); }
};
__device__ __forceinline__ int tiles_of(const Record& r) { return (r.kb_end - r.kb0 + NBLK - 1) / NBLK; }

// Value d of key `key` of a record's sequence and head, in units of v_scale; for the rows that see an infinity or a NaN.
template <int SRC>
__device__ __forceinline__ float value_at(const PromptParams& P, int b, int kvh, long long first_row, int key, int d) {
  if constexpr (SRC == kSrcPacked) {
    return __bfloat162float(P.v[(first_row + key) * P.v_token_stride + kvh * kHeadDim + d]);
  } else {
    const long long blk = P.block_table ? (long long)P.block_table[(size_t)b * P.max_blocks_per_seq + key / kBlock]
                                        : (long long)b * P.max_blocks_per_seq + key / kBlock;
    if (blk < 0 || blk >= P.num_blocks) return 0.f;
    const long long row = blk * P.Hkv + kvh;
    const int t = key % kBlock;
    if constexpr (SRC == kSrcBf16) {
      return __bfloat162float(static_cast<const __nv_bfloat16*>(P.v_cache)[(row * kBlock + t) * kHeadDim + d]);
    } else if constexpr (SRC == kSrcFp8) {
      return f16_lo_to_f32(e4m3x2_to_f16x2(static_cast<const uint8_t*>(P.v_cache)[(row * kBlock + t) * kHeadDim + d]));
    } else {   // only its scale can be a NaN
      const uint8_t* base = static_cast<const uint8_t*>(P.v_cache) + row * kFp4BlockBytes;
      return f16_lo_to_f32(e4m3x2_to_f16x2(base[fp4_v_scale_at(t, d >> 4)]));
    }
  }
}

// Whether every token of the record sees every key of tile t.
__device__ __forceinline__ bool all_see(const Record& r, int t, int window) {
  const int k0 = (r.kb0 + t * NBLK) * kBlock;
  return k0 + TK <= r.pos0 + 1 && (window == 0 || k0 >= r.pos0 + r.ntok - window);
}

// Row (block, KV head) of the cache that holds block j of a record's sequence; -1: outside the record's keys, or none (flagged).
__device__ __forceinline__ int cache_row(const PromptParams& P, const Record& r, int j) {
  if (j >= r.kb_end) return -1;
  const long long blk = P.block_table ? (long long)P.block_table[(size_t)r.b * P.max_blocks_per_seq + j]
                                      : (long long)r.b * P.max_blocks_per_seq + j;
  if (blk >= 0 && blk < P.num_blocks) return (int)(blk * P.Hkv + r.kvh);
  if (P.dev_status) atomicOr(P.dev_status, (int)PUZZLE_DEV_BAD_BLOCK);
  return -1;
}

}  // namespace

template <int SRC, int ROWS>
__global__ void __launch_bounds__(Cfg<SRC, ROWS>::kThreads, 1) prompt_attn_kernel(const __grid_constant__ PromptParams P) {
  using K = Cfg<SRC, ROWS>;
  constexpr int NS = K::kStages;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  uint8_t* smem = smem_raw + (((raw + 1023u) & ~1023u) - raw);
  Ctl* C = reinterpret_cast<Ctl*>(smem + K::kSmem);
  const uint32_t q_at = smem_u32(smem), k_at = q_at + ROWS * kTileBytes, v_at = k_at + NS * kTileBytes;
  [[maybe_unused]] const uint32_t code_at = v_at + NS * kTileBytes;
  const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;   // (uniform, as the compiler sees it)
  const int turns = ROWS == 1 ? 4 : P.turns, window = P.window;
  const Waiter wait{C, P.dev_status};

  if (warp == 0) {   // lane i: the i-th of every kind
    const int users = turns == 4 ? 2 : 4;   // streams that read a tile of keys
    if (lane < kRing) {
      mbar_init(smem_u32(&C->rec_full[lane]), 1);
      mbar_init(smem_u32(&C->rec_empty[lane]), 16 + 4 + 1 + 1 + (K::kPaged ? 4 : 0) + (K::kCodes ? 1 : 0));
    }
    if (lane < NS) {
      mbar_init(smem_u32(&C->k_full[lane]), K::kFullArrivals);
      mbar_init(smem_u32(&C->v_full[lane]), K::kFullArrivals);
      mbar_init(smem_u32(&C->k_empty[lane]), users);
      mbar_init(smem_u32(&C->v_empty[lane]), users);
      mbar_init(smem_u32(&C->v_ok[lane]), 1);
    }
    if (lane < 4) {
      mbar_init(smem_u32(&C->q_full[lane]), 1);
      mbar_init(smem_u32(&C->q_empty[lane]), turns);
      mbar_init(smem_u32(&C->join_full[lane]), 4 * turns);
      mbar_init(smem_u32(&C->s_full[lane]), 1);
      mbar_init(smem_u32(&C->p_full[lane]), 4);
      mbar_init(smem_u32(&C->ended[lane]), 1);
      mbar_init(smem_u32(&C->o_full[lane]), 1);
      mbar_init(smem_u32(&C->o_empty[lane]), 4 * turns);   // the warps that join
    }
    mbar_init(smem_u32(&C->copied[0][0] + lane), K::kCodes ? 1 : 32);
    if (lane < 8) mbar_init(smem_u32(&C->codes_empty[lane]), 4);
    if (lane == 0) {
      mbar_init(smem_u32(&C->next_full), 1);
      C->abort = 0;
      tma_prefetch_desc(&P.tmQ);
      if constexpr (!K::kPaged) {
        tma_prefetch_desc(&P.tmK);
        tma_prefetch_desc(&P.tmV);
      }
    }
    fence_mbar_init();
  }
  if (warp == 16) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&C->tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_before();
  __syncthreads();
  tc_after();
  const uint32_t tmem = __shfl_sync(kFull, C->tmem, 0);
  grid_dependency_wait();

  // The record of item n, copied; the slot is let go at once by those that do not need it later (release()).
  auto get_record = [&](int n, Record& r) -> bool {
    const int s = n % kRing;
    if (!wait(C->rec_full[s], (uint32_t)(n / kRing) & 1u)) return false;
    // the same in all lanes, and known to be: operands of MMAs and copies that come of it stay in uniform registers
    const Record& c = C->rec[s];
    r.on = __shfl_sync(kFull, c.on, 0);
    r.b = __shfl_sync(kFull, c.b, 0);
    r.kvh = __shfl_sync(kFull, c.kvh, 0);
    r.row0 = __shfl_sync(kFull, c.row0, 0);
    r.ntok = __shfl_sync(kFull, c.ntok, 0);
    r.pos0 = __shfl_sync(kFull, c.pos0, 0);
    r.kb0 = __shfl_sync(kFull, c.kb0, 0);
    r.kb_end = __shfl_sync(kFull, c.kb_end, 0);
    r.part = __shfl_sync(kFull, c.part, 0);
    return r.on != 0;
  };
  auto release = [&](int n) {
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&C->rec_empty[n % kRing]));
  };

  if (warp >= 16) {
    regs_down<K::kRegsOther>();
    if (warp < 20) {
      // ================================================================= MMA issue, one warp per stream
      const int st = warp - 16, tile = st / turns;
      constexpr uint32_t kFmt = K::kCodes ? 0u : 1u;   // P and V: f16 or bf16
      constexpr uint32_t kIdescQK = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24);
      constexpr uint32_t kIdescPV = (1u << 4) | (kFmt << 7) | (kFmt << 10) | (1u << 16) | (8u << 17) | (8u << 24);
      const uint32_t ts = tmem + kTmemS + 64 * st, to = tmem + kTmemO + 64 * st;
      const uint32_t q_lo = ((q_at + tile * kTileBytes) >> 4) + kDescLo, k_lo = (k_at >> 4) + kDescLo, v_lo = (v_at >> 4) + kDescLo;
      int base = 0, n = 0, items = 0, queries = 0;   // tiles of the items before; half tiles, items and query tiles of this stream
      Record r;
      bool ok = true;
      for (int it = 0; ok && get_record(it, r); ++it) {
        release(it);
        const Share sh(r, st, turns, window);
        if (sh.any()) {
          ok = wait(C->q_full[tile], (uint32_t)queries & 1u);
          ++queries;
          if (ok && !sh.on() && lane == 0) mbar_arrive(smem_u32(&C->q_empty[tile]));
        }
        const int nt = tiles_of(r);
        auto parity = [&](int t) { return (uint32_t)((base + t) / NS) & 1u; };
        auto skip = [&](int from, int to) {           // others' alone: let go of them
          for (int t = from; ok && t < to; ++t) {
            if (turns == 4 && (t & 1) != (st >> 1)) continue;   // two other streams' tile
            const int s = (base + t) % NS;
            ok = wait(C->k_full[s], parity(t)) && wait(C->v_ok[s], parity(t));
            if (ok && lane == 0) {
              mbar_arrive(smem_u32(&C->k_empty[s]));
              mbar_arrive(smem_u32(&C->v_empty[s]));
            }
            __syncwarp();
          }
        };
        skip(0, sh.on() ? sh.j0 >> 1 : nt);
        if (sh.on()) {
          // S of half tile j and its signals; the half tile after which a tile is let go of: the stream's last one in it.
          auto done = [&](int j) { return turns > 1 || (j & 1) || sh.last(j); };
          auto logits = [&](int j) {
            const int s = (base + (j >> 1)) % NS, nb = sh.blocks(j);
            const uint32_t k = k_lo + (uint32_t)(s * (kTileBytes / 16) + (j & 1) * (kTileBytes / 32));
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              umma_ss(ts, desc128(q_lo + 2 * ks), desc128(k + 2 * ks), kIdescQK | (uint32_t)(2 * nb) << 17, ks);
            umma_commit(smem_u32(&C->s_full[st]));
            if (done(j)) umma_commit(smem_u32(&C->k_empty[s]));
            if (sh.last(j)) umma_commit(smem_u32(&C->q_empty[tile]));
          };
          int j = sh.j0;
          ok = ok && wait(C->k_full[(base + (j >> 1)) % NS], parity(j >> 1));
          if (ok) {
            tc_after();
            if (elect_one()) logits(j);
            __syncwarp();
          }
          for (; ok && j < sh.j_hi; j += turns, ++n) {
            const int s = (base + (j >> 1)) % NS, nb = sh.blocks(j), next = j + turns;
            const bool first = j == sh.j0, more = next < sh.j_hi;
            // all that can be looked at before the weights are
            const uint64_t& k_next = C->k_full[(base + (next >> 1)) % NS];
            ok = wait(C->v_ok[s], parity(j >> 1)) && (!first || wait(C->o_empty[st], ((uint32_t)items & 1u) ^ 1u));
            const bool early = ok && more && __all_sync(kFull, mbar_test(smem_u32(&k_next), parity(next >> 1)));
            ok = ok && wait(C->p_full[st], (uint32_t)n & 1u);
            if (!ok) break;
            tc_after();
            if (elect_one()) {
              const uint32_t v = v_lo + (uint32_t)(s * (kTileBytes / 16) + (j & 1) * (kTileBytes / 32));
#pragma unroll
              for (int ks = 0; ks < kHalf; ++ks)   // a block of 16 keys each
                if (ks < nb) umma_ts(to, ts + 8 * ks, desc128(v + 128 * ks), kIdescPV, !(first && ks == 0));
              if (done(j)) umma_commit(smem_u32(&C->v_empty[s]));
              if (!more) umma_commit(smem_u32(&C->o_full[st]));
              // The next S overwrites this P.  Two products with different accumulators are not bound to run in the order of their
              // issue; what is issued before a fence::before_thread_sync is ordered before all tcgen05 operations behind it.
              tc_before();
              if (early) {
                tc_after();
                logits(next);
              }
            }
            __syncwarp();
            if (more && !early) {
              ok = wait(k_next, parity(next >> 1));
              if (!ok) break;
              tc_after();
              if (elect_one()) logits(next);
              __syncwarp();
            }
          }
          if (ok) skip(((sh.j_hi - 1 - ((sh.j_hi - 1 - sh.j0) & (turns - 1))) >> 1) + 1, nt);
          ++items;
        }
        base += nt;
      }
    } else if (warp == 20) {
      // ================================================================= work records, queries, packed keys and values
      const int T = kRowTokens * (4 / turns);
      const int per_tile = P.Hkv * P.splits;
      int b0 = 0, before = 0;           // a window of 32 sequences and the tiles of those before it
      int cnt = 0, upto = 0, st = 0, len = 0, ntok = 0;
      auto load_window = [&]() {
        const int b = b0 + lane;
        cnt = st = len = ntok = 0;
        if (b < P.batch) {
          st = P.starts[b];
          const int en = P.starts[b + 1];
          if (st >= 0 && en >= st && en <= P.total) ntok = en - st;
          else if (P.dev_status) atomicOr(P.dev_status, (int)PUZZLE_DEV_BAD_STARTS);
          len = ntok;
          if constexpr (K::kPaged) {
            if (ntok > 0) {
              len = P.seq_lens[b];
              const int most = P.max_blocks_per_seq * kBlock;
              if (len > most) {
                len = most;
                if (P.dev_status) atomicOr(P.dev_status, (int)PUZZLE_DEV_SEQ_TOO_LONG);
              }
              len = max(len, 0);
            }
          }
          cnt = (ntok + T - 1) / T;
        }
        upto = cnt;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int u = __shfl_up_sync(kFull, upto, d);
          if (lane >= d) upto += u;
        }
      };
      load_window();
      int it = 0, kt = 0, before_tiles = 0;
      bool ok = true;
      for (;; ++it) {
        // blocks of the grid are items, long ones first; a long one is asked for when the one before the last has been done with
        int item = blockIdx.x;
        const int slot = it % kRing;
        ok = wait(C->rec_empty[slot], ((uint32_t)(it / kRing) & 1u) ^ 1u);
        if (ok && it > 1 && before_tiles > kShortTiles)
          ok = wait(C->rec_empty[(it - 2) % kRing], (uint32_t)((it - 2) / kRing) & 1u);
        if (ok && it > 0) {
          fence_proxy_async();
          __syncwarp();
          if (elect_one()) {
            const uint32_t bar = smem_u32(&C->next_full);
            mbar_arrive_expect_tx(bar, 16);
            request_block(smem_u32(&C->next), bar);
          }
          __syncwarp();
          ok = wait(C->next_full, (uint32_t)(it - 1) & 1u);
          if (ok) item = granted_block(smem_u32(&C->next));
        }
        if (!ok) break;
        const int tile = item >= 0 ? item / per_tile : 0x7fffffff, rest = item - tile * per_tile;
        if (tile < before) {   // (blocks are granted in order; this does not rely on it)
          b0 = before = 0;
          load_window();
        }
        while (b0 < P.batch && before + __shfl_sync(kFull, upto, 31) <= tile) {
          before += __shfl_sync(kFull, upto, 31);
          b0 += 32;
          if (b0 < P.batch) load_window();
        }
        Record r;
        r.on = b0 < P.batch;
        r.b = r.kvh = r.row0 = r.ntok = r.pos0 = r.kb0 = r.kb_end = r.part = r.bad_v = 0;
        if (r.on) {
          const int src = __ffs(__ballot_sync(kFull, before + upto > tile)) - 1;
          const int s_cnt = __shfl_sync(kFull, cnt, src), s_upto = __shfl_sync(kFull, upto, src);
          const int s_st = __shfl_sync(kFull, st, src), s_len = __shfl_sync(kFull, len, src);
          const int s_n = __shfl_sync(kFull, ntok, src);
          const int i = s_cnt - 1 - (tile - (before + s_upto - s_cnt));   // a sequence's last tokens first
          r.b = b0 + src;
          r.kvh = rest % P.Hkv;
          r.part = rest / P.Hkv;
          r.row0 = s_st + i * T;
          r.ntok = min(T, s_n - i * T);
          r.pos0 = s_len - s_n + i * T;
          const int hi = max(r.pos0 + r.ntok, 0), lo = window > 0 ? max(r.pos0 - window + 1, 0) : 0;
          const int kb_hi = (hi + kBlock - 1) / kBlock, kb_lo = hi > 0 ? lo / kBlock : 0;
          const int nt = (kb_hi - kb_lo + NBLK - 1) / NBLK;
          const int parts = min(P.splits, max(nt, 1));
          if (r.part < parts) {
            r.kb0 = kb_lo + (int)((long long)nt * r.part / parts) * NBLK;
            r.kb_end = min(kb_lo + (int)((long long)nt * (r.part + 1) / parts) * NBLK, kb_hi);
          }
        }
        before_tiles = tiles_of(r);
        if (lane == 0) {
          C->rec[slot] = r;
          mbar_arrive(smem_u32(&C->rec_full[slot]));
        }
        __syncwarp();
        if (!r.on) break;
        if constexpr (!K::kPaged) {
          const int first = r.row0 - r.pos0;   // the sequence's first row
          const int nt = tiles_of(r);
          for (int t = 0; ok && t < nt; ++t, ++kt) {
            const int s = kt % NS;
            const uint32_t par = ((uint32_t)(kt / NS) & 1u) ^ 1u;
            const int row = first + (r.kb0 + t * NBLK) * kBlock;
            ok = wait(C->k_empty[s], par);
            if (ok && elect_one()) {
              const uint32_t bar = smem_u32(&C->k_full[s]);
              mbar_arrive_expect_tx(bar, kTileBytes);
              tma_load_3d(k_at + s * kTileBytes, &P.tmK, 0, r.kvh, row, bar);
            }
            __syncwarp();
            ok = ok && wait(C->v_empty[s], par);
            if (ok && elect_one()) {
              const uint32_t bar = smem_u32(&C->v_full[s]);
              mbar_arrive_expect_tx(bar, kTileBytes);
              tma_load_3d(v_at + s * kTileBytes, &P.tmV, 0, r.kvh, row, bar);
            }
            __syncwarp();
          }
        }
        if (!ok) break;
      }
      if (lane == 0) {
        C->asked = it;
        C->loaded = kt;
      }
    } else if (warp == 21) {
      // ================================================================= infinities and NaN among values not all rows see
      constexpr uint32_t kInf = K::kCodes ? 0x7c007c00u : 0x7f807f80u;
      int kt = 0;
      Record r;
      bool ok = true;
      for (int it = 0; ok && get_record(it, r); ++it) {
        const int nt = tiles_of(r);
        for (int t = 0; t < nt; ++t, ++kt) {
          const int s = kt % NS;
          ok = wait(C->v_full[s], (uint32_t)(kt / NS) & 1u);
          if (!ok) break;
          if (!all_see(r, t, window)) {
            const int nb = min(r.kb_end - r.kb0 - t * NBLK, NBLK);
            const uint32_t base = v_at + s * kTileBytes + 16 * lane;
            bool bad = false;
#pragma unroll 8
            for (int i = 0; i < nb * 4; ++i) {   // 512 bytes, four tokens each
              uint4 v = ld_shared16(base + 512 * i);
              const uint32_t x = __vcmpeq2(v.x & kInf, kInf), y = __vcmpeq2(v.y & kInf, kInf), z = __vcmpeq2(v.z & kInf, kInf),
                             u = __vcmpeq2(v.w & kInf, kInf);
              if (x | y | z | u) {
                bad = true;
                st_shared16(base + 512 * i, v.x & ~x, v.y & ~y, v.z & ~z, v.w & ~u);
              }
            }
            if (bad) {
              *reinterpret_cast<volatile int*>(&C->rec[it % kRing].bad_v) = 1;
              __threadfence_block();
              fence_proxy_async();
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&C->v_ok[s]));
        }
        release(it);
      }
    } else if (warp == 22) {
      // ================================================================= queries
      int q_n[4] = {0, 0, 0, 0};
      Record r;
      bool ok = true;
      for (int it = 0; ok && get_record(it, r); ++it) {
        release(it);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (!ok || i * turns >= 4 || !Share(r, i * turns, turns, window).any()) continue;
          ok = wait(C->q_empty[i], ((uint32_t)q_n[i] & 1u) ^ 1u);
          if (!ok) continue;
          ++q_n[i];
          if (elect_one()) {
            const uint32_t bar = smem_u32(&C->q_full[i]);
            mbar_arrive_expect_tx(bar, kTileBytes);
            tma_load_3d(q_at + i * kTileBytes, &P.tmQ, 0, r.kvh * kGroup, r.row0 + kRowTokens * i, bar);
          }
          __syncwarp();
        }
      }
      if (lane == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) C->q_loaded[i] = q_n[i];
    } else if (K::kCodes && warp == 23) {
      // ================================================================= codes of the cache, as they lie there
      // One lane to a block of K or V of a tile; places in the cache are looked up for four tiles at a time, lane = 8 tile + block.
      if constexpr (K::kCodes) {
        int in = 0;
        Record r;
        bool ok = true;
        for (int it = 0; ok && get_record(it, r); ++it) {
          release(it);
          const int nt = tiles_of(r);
          int row = -1;
          for (int t = 0; ok && t < nt; ++t, ++in) {
            if ((t & 3) == 0) row = cache_row(P, r, r.kb0 + t * NBLK + lane);
            const int mine = __shfl_sync(kFull, row, 8 * (t & 3) + ((lane & 15) >> 1)), slot = in % K::kCopySlots;
            ok = wait(C->codes_empty[slot], ((uint32_t)(in / K::kCopySlots) & 1u) ^ 1u);
            if (!ok) break;
            const uint32_t to = code_at + slot * K::kCodeTile + (((lane & 1) * NBLK + ((lane & 15) >> 1))) * K::kBlockBytes;
            const uint32_t bar = smem_u32(&C->copied[0][slot]);
            const uint32_t there = __ballot_sync(kFull, lane < 16 && mine >= 0);
            if (lane < 16 && mine < 0)   // no such block: zeros
              for (int i = 0; i < K::kBlockBytes / 16; ++i) st_shared16(to + 16 * i, 0, 0, 0, 0);
            __syncwarp();
            if (lane == 0) {
              if (there) mbar_arrive_expect_tx(bar, __popc(there) * K::kBlockBytes);
              else mbar_arrive(bar);
            }
            __syncwarp();
            if (there >> lane & 1u)
              bulk_copy(to, static_cast<const char*>(lane & 1 ? P.v_cache : P.k_cache) + (size_t)mine * K::kBlockBytes, K::kBlockBytes,
                        bar);
            __syncwarp();
          }
        }
        for (int i = max(in - K::kCopySlots, 0); i < in; ++i)
          mbar_wait_bounded(smem_u32(&C->copied[0][i % K::kCopySlots]), (uint32_t)(i / K::kCopySlots) & 1u);
      }
    } else if (K::kPaged && warp >= 24) {
      // ================================================================= tiles of the cache in the MMAs' form, four warps
      // Warp lw has blocks lw and lw + 4 of every tile, K and V.
      const int lw = warp - 24;
      if constexpr (SRC == kSrcBf16) {
      // Copied to where the MMAs read them.  Places in the cache are looked up for 16 tiles at a time, lane = 2 tile + block.
      constexpr int kSlots = K::kCopySlots;
      auto lookup = [&](const Record& r, int t_first) { return cache_row(P, r, r.kb0 + (t_first + (lane >> 1)) * NBLK + lw + 4 * (lane & 1)); };
      bool ok = true;
      // The next tile to copy.  Records of items that nothing is copied of yet are taken only as they come: their being
      // published can depend on tiles that this warp has still to hand on.
      Record r;
      int it = -1, t = 0, nt = 0, ent = -1;
      bool more = true;
      auto have_tile = [&](bool block) -> bool {
        while (more && t == nt) {
          const int s = (it + 1) % kRing;
          const uint32_t par = (uint32_t)((it + 1) / kRing) & 1u;
          if (!block && !__all_sync(kFull, mbar_try_wait(smem_u32(&C->rec_full[s]), par))) return false;
          more = get_record(it + 1, r);
          if (!more) return false;
          release(++it);
          t = 0;
          nt = tiles_of(r);
          if (nt > 0) ent = lookup(r, 0);
        }
        return more;
      };
      int in = 0, out = 0;                         // tiles whose copies are begun, tiles handed on
      auto begin_copy = [&]() {
        const int row0 = __shfl_sync(kFull, ent, 2 * (t & 15)), row1 = __shfl_sync(kFull, ent, 2 * (t & 15) + 1);
        const int s = in % NS;
        const uint32_t par = ((uint32_t)(in / NS) & 1u) ^ 1u;
        ok = wait(C->k_empty[s], par) && wait(C->v_empty[s], par);
        if (!ok) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int row = h ? row1 : row0;
          const size_t at = (size_t)max(row, 0) * (kBlock * kHeadDim * 2);
          const char* ks = static_cast<const char*>(P.k_cache) + at;
          const char* vs = static_cast<const char*>(P.v_cache) + at;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int cidx = lane + 32 * i, tok = (lw + 4 * h) * kBlock + (cidx >> 3);
            const uint32_t dst = (uint32_t)(s * kTileBytes + tok * 128 + (((cidx & 7) ^ (tok & 7)) << 4));
            cp_async16(k_at + dst, ks + 16 * cidx, row >= 0);
            cp_async16(v_at + dst, vs + 16 * cidx, row >= 0);
          }
        }
        cp_arrive(smem_u32(&C->copied[lw][in % kSlots]));
        ++in;
        if (++t < nt && (t & 15) == 0) ent = lookup(r, t);
      };
      while (ok) {
        while (ok && in - out < kSlots && have_tile(in == out)) begin_copy();
        if (!ok || in == out) break;
        ok = wait(C->copied[lw][out % kSlots], (uint32_t)(out / kSlots) & 1u);
        if (!ok) break;
        const int s = out % NS;
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(smem_u32(&C->k_full[s]));
          mbar_arrive(smem_u32(&C->v_full[s]));
        }
        ++out;
      }
      cp_wait_all();
     } else if constexpr (K::kCodes) {
      // Codes of a tile -> bf16 keys and f16 values in the swizzled rows that the MMAs read.
      auto convert = [&](uint32_t src, uint32_t dst, bool is_v) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int blk = lw + 4 * h;
          const uint32_t cb = src + blk * K::kBlockBytes;
          if constexpr (SRC == kSrcFp8) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int cidx = lane + 32 * i, tok = blk * kBlock + (cidx >> 2), o = 2 * (cidx & 3);
              const uint4 w4 = ld_shared16(cb + 16 * cidx);
              const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
              uint32_t x[8];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                x[2 * k] = e4m3x2_to_f16x2(w[k] & 0xffffu);
                x[2 * k + 1] = e4m3x2_to_f16x2(w[k] >> 16);
              }
              if (!is_v)
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = f16x2_to_bf16x2(x[k]);
              const uint32_t row = dst + tok * 128;
              st_shared16(row + ((o ^ (tok & 7)) << 4), x[0], x[1], x[2], x[3]);
              st_shared16(row + (((o + 1) ^ (tok & 7)) << 4), x[4], x[5], x[6], x[7]);
            }
          } else if constexpr (SRC == kSrcFp4) {
            const uint4 w4 = ld_shared16(cb + 16 * lane);
            const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
            auto scale2 = [&](int at) -> __half2 {   // the E4M3 scale at this byte of the block, twice
              uint32_t sc;
              asm volatile("ld.shared.u8 %0, [%1];" : "=r"(sc) : "r"(cb + at) : "memory");
              const uint32_t hh = e4m3x2_to_f16x2(sc | (sc << 8));
              return *reinterpret_cast<const __half2*>(&hh);
            };
            auto times = [](uint32_t a, __half2 s) -> uint32_t {
              const __half2 p = __hmul2(*reinterpret_cast<const __half2*>(&a), s);
              return *reinterpret_cast<const uint32_t*>(&p);
            };
            if (!is_v) {   // token lane / 2, channels 32 (lane % 2) ..
              const int t = lane >> 1, tok = blk * kBlock + t, g = 2 * (lane & 1);
              const uint32_t row = dst + tok * 128;
#pragma unroll
              for (int k = 0; k < 4; ++k) {   // eight channels
                const __half2 sc = scale2(fp4_k_scale_at(t, g + (k >> 1)));
                uint32_t x0, x1, x2, x3;
                e2m1x8_to_f16x2x4(w[k], x0, x1, x2, x3);
                st_shared16(row + (((2 * g + k) ^ (tok & 7)) << 4), f16x2_to_bf16x2(times(x0, sc)), f16x2_to_bf16x2(times(x1, sc)),
                            f16x2_to_bf16x2(times(x2, sc)), f16x2_to_bf16x2(times(x3, sc)));
              }
            } else {       // tokens 2 tp and 2 tp + 1, channels 32 (lane / 16) + 16 (lane % 2) ..
              const int tp = (lane & 15) >> 1, g = 2 * (lane >> 4) + (lane & 1), tok = blk * kBlock + 2 * tp;
              const __half2 s0 = scale2(fp4_v_scale_at(2 * tp, g)), s1 = scale2(fp4_v_scale_at(2 * tp + 1, g));
              const uint32_t row = dst + tok * 128;
#pragma unroll
              for (int k = 0; k < 2; ++k) {   // eight channels of both tokens
                uint32_t e[4], o[4];
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                  uint32_t x0, x1, x2, x3;   // (even token, odd token) of four channels
                  e2m1x8_to_f16x2x4(w[2 * k + m], x0, x1, x2, x3);
                  e[2 * m] = times(prmt(x0, x1, 0x5410), s0);
                  e[2 * m + 1] = times(prmt(x2, x3, 0x5410), s0);
                  o[2 * m] = times(prmt(x0, x1, 0x7632), s1);
                  o[2 * m + 1] = times(prmt(x2, x3, 0x7632), s1);
                }
                st_shared16(row + (((2 * g + k) ^ (tok & 7)) << 4), e[0], e[1], e[2], e[3]);
                st_shared16(row + 128 + (((2 * g + k) ^ ((tok + 1) & 7)) << 4), o[0], o[1], o[2], o[3]);
              }
            }
          }
        }
      };
      auto signal = [&](const uint64_t& bar) {
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bar));
      };
      int n = 0;
      Record r;
      bool ok = true;
      for (int it = 0; ok && get_record(it, r); ++it) {
        release(it);
        const int nt = tiles_of(r);
        for (int t = 0; t < nt; ++t, ++n) {
          const int s = n % NS, slot = n % K::kCopySlots;
          const uint32_t par = ((uint32_t)(n / NS) & 1u) ^ 1u, src = code_at + slot * K::kCodeTile;
          ok = wait(C->copied[0][slot], (uint32_t)(n / K::kCopySlots) & 1u) && wait(C->k_empty[s], par);
          if (!ok) break;
          convert(src, k_at + s * kTileBytes, false);
          signal(C->k_full[s]);
          ok = wait(C->v_empty[s], par);
          if (!ok) break;
          convert(src + NBLK * K::kBlockBytes, v_at + s * kTileBytes, true);
          signal(C->v_full[s]);
          if (lane == 0) mbar_arrive(smem_u32(&C->codes_empty[slot]));
        }
      }
     }
    }
    sync_cta();
    if (C->abort) {   // what is still under way ends before shared and tensor memory are given back
      if (warp < 20) {
        if (elect_one()) umma_commit(smem_u32(&C->ended[warp - 16]));
        __syncwarp();
        mbar_wait_bounded(smem_u32(&C->ended[warp - 16]), 0);
      } else if (warp == 20) {
        const int it = C->asked, kt = C->loaded;
        if (it > 0) mbar_wait_bounded(smem_u32(&C->next_full), (uint32_t)(it - 1) & 1u);
#pragma unroll 1
        for (int i = max(kt - NS, 0); i < kt; ++i) {
          mbar_wait_bounded(smem_u32(&C->k_full[i % NS]), (uint32_t)(i / NS) & 1u);
          mbar_wait_bounded(smem_u32(&C->v_full[i % NS]), (uint32_t)(i / NS) & 1u);
        }
      } else if (warp == 22) {
#pragma unroll 1
        for (int i = 0; i < 4; ++i)
          if (C->q_loaded[i] > 0) mbar_wait_bounded(smem_u32(&C->q_full[i]), (uint32_t)(C->q_loaded[i] - 1) & 1u);
      }
      __syncwarp();
    }
  } else {
    // =================================================================== softmax, four warpgroups, thread = row
    regs_up<K::kRegsSoftmax>();
    const int st = warp >> 2, tile = st / turns, wq = warp & 3, row = 32 * wq + lane;
    const uint32_t quad = (uint32_t)(32 * wq) << 16;
    const uint32_t ts = tmem + kTmemS + 64 * st + quad, to = tmem + kTmemO + quad;
    const bool wide_out = (reinterpret_cast<uintptr_t>(P.out) & 31) == 0;   // 32 bytes of a row in one store
    int n = 0, items = 0;   // half tiles and items of this stream
    Record r;
    bool ok = true;
    for (int it = 0; ok && get_record(it, r); ++it) {
      const Share sh(r, st, turns, window);
      float scale = P.sm_scale_log2e;
      if (K::kCodes && P.k_scale) scale *= P.k_scale[r.kvh];
      // scaled: this row's logits are scaled before their maximum is taken; odd: some row's of this warp
      bool odd = !(scale > 0.f && scale < INFINITY), scaled = odd;
      const int p = sh.pos + (row >> 3), p0 = sh.pos + 4 * wq; // this row's position, the warp's first
      const int hi = p + 1, lo = window > 0 ? p - window + 1 : 0;   // the row sees [lo, hi)
      // Rows without a token hold what is behind the sequence: other sequences' queries, and logits from earlier items.  They do not
      // take part in what a warp decides together, so that these change no bit of a result.
      const bool real = (row >> 3) < sh.ntok;
      float ref = kUnset, l = 0.f;                             // weights are 2^(c s - ref)
      for (int j0 = sh.j0; j0 < sh.j_hi; j0 += turns, ++n) {
        const int nb = sh.blocks(j0), k0 = (r.kb0 + j0 * kHalf) * kBlock;
        ok = wait(C->s_full[st], (uint32_t)n & 1u);
        if (!ok) break;
        tc_after();
        bool done = false;
        if (j0 != sh.j0 && !odd && k0 + TK / 2 <= p0 + 1 && (window == 0 || k0 >= p0 + 3 - window + 1)) {
          // The usual half tile: every token of this warp sees all 64 keys, and their weights are in bounds.
          uint32_t u[64];
          const float* s = reinterpret_cast<const float*>(u);
          float big = 0.f;
          tmem_ld32(ts, u);
          tmem_ld32(ts + 32, u + 32);
          tmem_wait_ld();
          const uint64_t c2 = pack2(scale, scale), r2 = pack2(-ref, -ref);
          uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            float x0, x1, e0, e1;
            const uint64_t x2 = fma2(pack2(s[2 * j], s[2 * j + 1]), c2, r2);
            unpack2(x2, x0, x1);
            if (j % 4 == 2) {   // a quarter of them on the FMA units
              big = max3(big, x0, x1);
              exp2_poly(x2, e0, e1);
            } else {
              e0 = ex2(x0);
              e1 = ex2(x1);
            }
            sum[j & 1] = add2(sum[j & 1], pack2(e0, e1));
            u[j] = K::kCodes ? f32x2_to_f16x2(e0, e1) : f32x2_to_bf16x2(e0, e1);
          }
          float a0, a1;
          unpack2(add2(sum[0], sum[1]), a0, a1);
          done = !__any_sync(kFull, real && (!(a0 + a1 < K::kMuch) || !(big < 100.f)));
          if (done) {
            l += a0 + a1;
            tmem_st32(ts, u);
          }
        }
        if (!done) {
        // 32 keys at a time.  P of the first 32 lies over their own logits.
#pragma unroll 1
        for (int q = 0; q < (nb > 2 ? 2 : 1); ++q) {
          const int kc = k0 + 32 * q;
          uint32_t y[16];
          if (kc > p0 + 3 || (window > 0 && kc + 32 <= p0 - window + 1)) {   // no token of this warp sees any of them
#pragma unroll
            for (int j = 0; j < 16; ++j) y[j] = 0u;
          } else {
            uint32_t u[32];
            float* s = reinterpret_cast<float*>(u);
            tmem_ld32(ts + 32 * q, u);
            tmem_wait_ld();
            if (odd || kc + 32 > p0 + 1 || (window > 0 && kc < p0 + 3 - window + 1)) {   // some token does not see some of them
              if (odd)
#pragma unroll
                for (int j = 0; j < 32; ++j) s[j] *= scaled ? scale : 1.f;
              const uint32_t seen = bits_below(p + 1 - kc) & ~(window > 0 ? bits_below(p - window + 1 - kc) : 0u);
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if (!(seen & (1u << j))) s[j] = -INFINITY;
            }
            float part;
            for (bool look = j0 == sh.j0 && q == 0;; look = true) {
              if (look) {
                float x[2] = {s[0], s[1]};   // NaN beats everything
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                  x[0] = max3(x[0], s[j], s[j + 1]);
                  x[1] = max3(x[1], s[j + 2], s[j + 3]);
                }
                float top = max3(x[0], x[1], x[1]), now = top * (scaled ? 1.f : scale) - K::kShift;
                // A weight is 2^(c s - ref) rounded once, so what rounding took from the reference is a factor of all of the row's
                // weights and falls out.  Beyond 2^20 that factor leaves the range of the weights: then the row's logits are scaled,
                // and rounded, first, the reference is the largest of them itself, and the differences are exact.
                const bool large = real && fabsf(top) < INFINITY && fabsf(now) > kLarge && !scaled;
                if (__any_sync(kFull, large)) {
                  odd = true;
                  const float by = large ? scale : 1.f;
#pragma unroll
                  for (int j = 0; j < 32; ++j) s[j] *= by;
                  top *= by;
                  scaled |= large;
                }
                if (scaled && fabsf(top) > kLarge) now = top;
                const bool raise = real && now > ref;
                if (__any_sync(kFull, raise)) {
                  float alpha = 1.f;
                  if (raise) {   // by whole powers of two: what was rounded before keeps its bits
                    const float up = now - ref > 128.f ? now : ref + ceilf(now - ref);   // (beyond 128 nothing is left of those)
                    alpha = ex2(ref - up);
                    ref = up;
                  }
                  __syncwarp();            // what follows goes through tensor memory by whole warps
                  l *= alpha;
                  if (q == 1) rescale_weights<K::kCodes>(ts, alpha);
                  if (j0 != sh.j0) {       // the product before has ended: this S was issued behind it
#pragma unroll 1
                    for (int i = 0; i < 4; ++i) {
                      uint32_t o[16];
                      tmem_ld16(to + 64 * st + 16 * i, o);
                      tmem_wait_ld();
#pragma unroll
                      for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha);
                      tmem_st16(to + 64 * st + 16 * i, o);
                    }
                  }
                }
                // infinity - infinity, or a NaN: the whole row is NaN
                ref = top < INFINITY ? ref : NAN;
              }
              const float c = scaled ? 1.f : scale;
              const uint64_t c2 = pack2(c, c), r2 = pack2(-ref, -ref);
              uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
              for (int j = 0; j < 16; ++j) {
                float x0, x1;
                unpack2(fma2(pack2(s[2 * j], s[2 * j + 1]), c2, r2), x0, x1);
                const float e0 = ex2(x0), e1 = ex2(x1);
                sum[j & 1] = add2(sum[j & 1], pack2(e0, e1));
                y[j] = K::kCodes ? f32x2_to_f16x2(e0, e1) : f32x2_to_bf16x2(e0, e1);
              }
              float a0, a1;
              unpack2(add2(sum[0], sum[1]), a0, a1);
              part = a0 + a1;
              if (look || !__any_sync(kFull, real && !(part < K::kMuch))) break;
            }
            l += part;
          }
          tmem_st16(ts + 16 * q, y);
        }
        }
        tmem_wait_st();
        tc_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&C->p_full[st]));
      }
      if (!ok) break;
      // ---- the item's end: the streams of a tile of rows join, each for its part of the channels
      const int g = r.kvh * kGroup + (row & 7);
      float sk = -INFINITY;                    // (asked for before the wait)
      if (P.splits == 1 && P.sinks) sk = P.sinks[g] * kLog2e;
      if (sh.on()) {
        ok = wait(C->o_full[st], (uint32_t)items & 1u);
        if (!ok) break;
        ++items;
      }
      if (ref == kUnset && l == 0.f) ref = -INFINITY;    // no logit above -inf
      const int g0 = st & ~(turns - 1), cols = 64 / turns, col0 = cols * (st - g0);
      const float own = ref;
      float own_l = l;
      if (turns > 1) {
        C->join[it & 1][st][row] = make_float2(ref, l);
        tc_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&C->join_full[tile]));
        ok = wait(C->join_full[tile], (uint32_t)it & 1u);
        if (!ok) break;
        for (int i = g0; i < g0 + turns; ++i) ref = fmaxf(ref, C->join[it & 1][i][row].x);
      }
      tc_after();
      const float zero = ref == -INFINITY ? 0.f : ref;
      l = 0.f;
      for (int i = g0; i < g0 + turns; ++i) {
        const float2 side = turns > 1 ? C->join[it & 1][i][row] : make_float2(own, own_l);
        l += side.y * ex2(side.x - zero);
      }
      const long long at = (r.row0 + kRowTokens * tile + (long long)(row >> 3)) * (P.Hkv * kGroup) + g;
      float z = l, big = ref;
      if (P.splits == 1 && P.sinks) {
        big = sk > ref ? sk : ref;             // a NaN sink is not above; it comes in through z
        const float base = big == -INFINITY ? 0.f : big;
        z = l * ex2(ref - base) + ex2(sk - base);
      }
      const float base = big == -INFINITY ? 0.f : big;
      float f = ex2(ref - base) * (K::kCodes && P.v_scale ? P.v_scale[r.kvh] : 1.f) / z;
      float lse = (base + lg2(z)) * kLn2;
      const size_t part_row = (size_t)r.part * ((size_t)P.total * (P.Hkv * kGroup)) + at;
      if (P.splits > 1) {
        if (l == 0.f) lse = -INFINITY;         // no key in this part, or none above -inf
        if (real && col0 == 0) P.part_lse[part_row] = lse;
      } else {
        if (z == 0.f) {                        // nothing seen: zeros; nothing but logits of -inf: 0 / 0
          f = hi > 0 ? NAN : 0.f;
          lse = hi > 0 ? NAN : -INFINITY;
        }
        if (real && P.lse_out && col0 == 0) P.lse_out[at] = lse;
      }
      const bool bad = *reinterpret_cast<volatile int*>(&C->rec[it % kRing].bad_v) != 0;
      uint32_t with = sh.on() ? 1u << st : 0u;   // the streams that have an O
      if (turns > 1)
        for (int i = g0; i < g0 + turns; ++i) with |= Share(r, i, turns, window).on() ? 1u << i : 0u;
#pragma unroll 1
      for (int c0 = col0; c0 < col0 + cols; c0 += 16) {
        __syncwarp();                            // tensor memory is read by whole warps; rows without a token store nothing
        float o[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) o[j] = 0.f;
#pragma unroll 1
        for (int i = g0; i < g0 + turns; ++i) {
          if (!(with >> i & 1u)) continue;
          const float a = ex2((turns > 1 ? C->join[it & 1][i][row].x : own) - zero);
          uint32_t v[16];
          tmem_ld16(to + 64 * i + c0, v);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 16; ++j) o[j] += __uint_as_float(v[j]) * a;
        }
        if (real && bad) {
          const int from = max(max(lo, 0), r.kb0 * kBlock), to_key = min(hi, r.kb_end * kBlock);
          const long long first_row = (long long)r.row0 - r.pos0;
          for (int key = from; key < to_key; ++key) {
            const int t = (key / kBlock - r.kb0) / NBLK;
            if (all_see(r, t, window)) {       // the product has them
              key = (r.kb0 + (t + 1) * NBLK) * kBlock - 1;
              continue;
            }
#pragma unroll 1
            for (int d = 0; d < 16; ++d) {
              const float v = value_at<SRC>(P, r.b, r.kvh, first_row, key, c0 + d);
              if (!(fabsf(v) < INFINITY)) {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                  if (j == d) o[j] += v;
              }
            }
          }
        }
        if (real && P.splits > 1) {
          if (lse != -INFINITY) {
            float4* dst = reinterpret_cast<float4*>(P.part_o + part_row * kHeadDim + c0);
#pragma unroll
            for (int j = 0; j < 4; ++j) dst[j] = make_float4(o[4 * j] * f, o[4 * j + 1] * f, o[4 * j + 2] * f, o[4 * j + 3] * f);
          }
        } else if (real) {
          uint32_t y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = f32x2_to_bf16x2(o[2 * j] * f, o[2 * j + 1] * f);
          __nv_bfloat16* dst = P.out + at * kHeadDim + c0;
          if (wide_out) {
            asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]),
                         "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7])
                         : "memory");
          } else {
            reinterpret_cast<uint4*>(dst)[0] = make_uint4(y[0], y[1], y[2], y[3]);
            reinterpret_cast<uint4*>(dst)[1] = make_uint4(y[4], y[5], y[6], y[7]);
          }
        }
      }
      __syncwarp();
      tc_before();
      if (lane == 0)
        for (int i = g0; i < g0 + turns; ++i)
          if (with >> i & 1u) mbar_arrive(smem_u32(&C->o_empty[i]));
      release(it);
      __syncwarp();
    }
    sync_cta();
  }
  if (C->abort) sync_cta();   // (no role is left that could set it)
  if (warp == 16) {
    __syncwarp();
    tc_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

namespace {

// Partials of the parts of a row -> its output; 16 lanes a row.
__global__ void __launch_bounds__(256) prompt_merge_kernel(const __grid_constant__ PromptParams P) {
  const int Hq = P.Hkv * kGroup;
  const size_t rows = (size_t)P.total * Hq;
  const size_t at = ((size_t)blockIdx.x * blockDim.x + threadIdx.x) >> 4;
  const int o = threadIdx.x & 15;
  grid_dependency_wait();
  if (at >= rows) return;
  const int token = (int)(at / Hq), g = (int)(at % Hq);
  const float* lse = P.part_lse + at;
  float top = P.sinks ? P.sinks[g] : -INFINITY;
  const float sk = top;
  for (int p = 0; p < P.splits; ++p) top = fmaxf(top, lse[p * rows]);
  const float base = top == -INFINITY ? 0.f : top;
  float z = P.sinks ? ex2((sk - base) * kLog2e) : 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p = 0; p < P.splits; ++p) {
    const float e = lse[p * rows];
    if (e == -INFINITY) continue;
    const float wgt = ex2((e - base) * kLog2e);
    const float4 v = reinterpret_cast<const float4*>(P.part_o + (p * rows + at) * kHeadDim)[o];
    z += wgt;
    acc.x += wgt * v.x;
    acc.y += wgt * v.y;
    acc.z += wgt * v.z;
    acc.w += wgt * v.w;
  }
  // The row's sequence: valid ones do not share rows, but with bad entries among them need not lie in order.
  const unsigned sixteen = 0xffffu << (threadIdx.x & 16);
  int seq = -1;
  for (int b = o; b < P.batch; b += 16) {
    const int st = P.starts[b], en = P.starts[b + 1];
    if (st >= 0 && st <= token && token < en && en <= P.total) seq = b;
  }
#pragma unroll
  for (int d = 8; d > 0; d >>= 1) seq = max(seq, __shfl_xor_sync(sixteen, seq, d));
  if (seq < 0) return;                  // no sequence's row: what was read of it means nothing
  const int len = min(max(P.seq_lens[seq], 0), P.max_blocks_per_seq * kBlock);
  const bool sees = len - (P.starts[seq + 1] - token) >= 0;
  float f = 1.f / z, out_lse = base + lg2(z) * kLn2;
  if (z == 0.f) {
    f = sees ? NAN : 0.f;
    out_lse = sees ? NAN : -INFINITY;
  }
  reinterpret_cast<uint2*>(P.out + at * kHeadDim)[o] = make_uint2(f32x2_to_bf16x2(acc.x * f, acc.y * f), f32x2_to_bf16x2(acc.z * f, acc.w * f));
  if (P.lse_out && o == 0) P.lse_out[at] = out_lse;
}

template <int SRC, int ROWS>
cudaError_t launch_as(const PromptParams& P, cudaStream_t s, int* smem_limit) {
  const int need = Cfg<SRC, ROWS>::kSmem + (int)sizeof(Ctl) + 1024;
  if (*smem_limit == 0) {
    const cudaError_t e = cudaFuncSetAttribute(prompt_attn_kernel<SRC, ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize, need);
    if (e != cudaSuccess) return e;
    *smem_limit = need;
  }
  const int T = kRowTokens * (4 / P.turns);
  const long long tiles = P.total / T + std::min(P.batch, P.total);   // no more than these, whatever the lengths
  const long long items = tiles * P.Hkv * P.splits;
  if (items > 0x7fffffff) return cudaErrorInvalidValue;
  cudaError_t e = launch_dependent(prompt_attn_kernel<SRC, ROWS>, dim3((unsigned)items),
                                   dim3(Cfg<SRC, ROWS>::kThreads), need, s, P);
  count_launch();
  if (e == cudaSuccess && P.splits > 1) {
    const size_t threads = (size_t)P.total * P.Hkv * kGroup * 16;
    e = launch_dependent(prompt_merge_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, P);
    count_launch();
  }
  return e;
}

template <int SRC>
cudaError_t launch(const PromptParams& P, cudaStream_t s, int* smem_limit) {
  return P.turns == 4 ? launch_as<SRC, 1>(P, s, smem_limit + 4) : launch_as<SRC, 4>(P, s, smem_limit);
}

}  // namespace

static long long groups_of(long long batch, long long total, int turns, int Hkv) {   // at least so many
  const long long T = kRowTokens * (4 / turns);
  return std::max<long long>((total + T - 1) / T, std::min(batch, total)) * Hkv;
}

// The size of a group (64, 32 or 16 tokens: 1, 2 or 4 streams to a tile of rows) and the parts that its keys are cut into: what takes
// the SM with the most items the least time, in steps of 64 keys of a stream.  A tile of keys is 2, 1 or 1/2 steps of each stream, and
// fetching it (converting it, for codes) some of a step whatever the group; an item costs about five steps beside its keys.  Parts
// have four tiles at least, and there are at most 4 items per SM where keys are cut, which bounds the partials.  (512 tokens over 64K
// E4M3 keys: groups of 16 uncut 1224 us, of 32 in 8 parts 849.)
// Where none of these numbers of parts leaves four tiles to a part, as many as do are taken, though they fill fewer SMs: one sequence, one KV
// head, 5 tokens over 65536 E4M3 keys uncut 534 us, in 128 parts 43; 8 KV heads, 9000 keys 81 and 23, 1500 keys 21 and 19.  (Keys
// are counted by the table's row: 300 of them in a row for 9000 take 13 us uncut, 16 in parts.)
PromptPlan prompt_plan(int batch, int total, int Hkv, long long key_bound, bool may_split, double fetch, int sm_count) {
  PromptPlan plan = {1, 4};
  double best = 1e30;
  for (int fewer = 0; fewer < 2 && plan.splits == 1; ++fewer)
    for (int turns = 1; turns <= 4; turns *= 2) {
      const long long items = groups_of(batch, total, turns, Hkv), T = kRowTokens * (4 / turns);
      const double tiles = std::max(1.0, (double)(key_bound + T) / TK);
      const long long most = (long long)(tiles / 4);
      for (int per_sm = 0; per_sm <= (may_split ? 4 : 0); ++per_sm) {   // uncut; as many parts as fill each SM once, twice ..
        long long n = per_sm == 0 ? 1 : per_sm * (long long)sm_count / items;
        if (fewer) n = std::min(n, most);
        if (n < 1 || (n > 1 && n > most)) continue;
        const double rounds = (double)((items * n + sm_count - 1) / sm_count);
        const double cost = rounds * (tiles / n * (2.0 / turns + fetch) + 5) + (n > 1 ? 4 : 0);
        if (cost < best * 0.98) {   // a little gain is not worth the partials
          best = cost;
          plan.splits = (int)n;
          plan.turns = turns;
        }
      }
    }
  return plan;
}

size_t prompt_partial_bytes(int total, int Hkv, int splits) {
  return std::max<size_t>(16, splits > 1 ? (size_t)splits * total * Hkv * kGroup * (kHeadDim + 1) * sizeof(float) : 0);
}
// The most parts that prompt_plan cuts into, whatever the context's length.
int prompt_most_splits(int batch, int total, int Hkv, int sm_count) {
  return (int)std::max<long long>(1, 4ll * sm_count / std::max<long long>(1, groups_of(batch, total, 1, Hkv)));
}

cudaError_t launch_prompt_attn(const PromptParams& P, PromptSource src, cudaStream_t s, int* smem_limit) {
  switch (src) {
    case kSrcPacked: return launch<kSrcPacked>(P, s, smem_limit + 0);
    case kSrcBf16: return launch<kSrcBf16>(P, s, smem_limit + 1);
    case kSrcFp8: return launch<kSrcFp8>(P, s, smem_limit + 2);
    default: return launch<kSrcFp4>(P, s, smem_limit + 3);
  }
}

}  // namespace puzzle
