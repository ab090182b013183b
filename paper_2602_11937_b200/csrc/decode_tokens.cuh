// Pairs of query tokens: which keys a pair sees, and the arithmetic of a pair over the 4-bit cache.  Include inside a
// translation unit only (internal linkage).
#pragma once

#include "common.cuh"
#include "decode_attn.cuh"
#include "decode_tile_fp4.cuh"

namespace puzzle {
namespace {

constexpr int kTokTile = 64;

// One row of the schedule: query tokens t0 and t1 (= t0 + 1, or t0 again for an odd last token) of sequence b.
struct RowInfo {
  int b, t0, t1;
  int L, LA;     // keys [lo, L) are visible to t1, [loA, LA) to t0 (LA = L - (t1 - t0))
  int lo, loA;
  int tlo, ntile;  // tiles that cover [loA, L)
  bool present, too_long;
};
__device__ __forceinline__ RowInfo row_info(const DecodeParams& P, int r) {
  RowInfo i;
  const int npairs = (P.n_q + 1) >> 1;
  i.b = r / npairs;
  const int j = r - i.b * npairs;
  const int qlen = P.q_lens ? max(0, min(P.q_lens[i.b], P.n_q)) : P.n_q;
  i.t0 = 2 * j;
  i.present = i.t0 < qlen;
  i.t1 = min(i.t0 + 1, qlen - 1);
  const int max_tokens = P.max_blocks_per_seq * kBlock;
  const int len = P.seq_lens[i.b];
  i.too_long = len > max_tokens;
  const int Lb = len < 0 ? 0 : min(len, max_tokens);
  i.L = i.present ? max(0, Lb - qlen + i.t1 + 1) : 0;
  i.LA = max(0, i.L - (i.t1 - i.t0));
  i.lo = (P.window > 0 && i.L > P.window) ? i.L - P.window : 0;
  i.loA = (P.window > 0 && i.LA > P.window) ? i.LA - P.window : 0;
  i.tlo = i.loA / kTokTile;
  i.ntile = i.L > 0 ? (i.L + kTokTile - 1) / kTokTile - i.tlo : 0;
  return i;
}

// Ones where a byte of four E4M3 values is a NaN.
__device__ __forceinline__ uint32_t e4m3_nans(uint32_t x) { return __vcmpeq4(x & 0x7f7f7f7fu, 0x7f7f7f7fu); }
__device__ __forceinline__ void sts32(uint32_t a, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }

struct Fp4Pair {
  using Tile = Fp4Tile;
  struct State {
    Fp4State t[2];
    __device__ __forceinline__ void reset() { t[0].reset(); t[1].reset(); }
  };
  static __device__ __forceinline__ void load_query(State& st, int tok, const __nv_bfloat16* qrow, float ks, float sm,
                                                    int lane) {
    st.t[tok].load_query(qrow, ks, sm, lane);
  }
  // A key that only one of the two tokens sees (the newest, the oldest of a window) meets the other's weight of zero in the
  // shared product, and a NaN among its V scales would make that a NaN.  Such a scale is cleared in shared memory, and the
  // channels it covers become NaN for the token that sees the key.  Nothing of this is live beside the tile's registers:
  // converting V once for each token instead costs 10 % of a long call (155 to 171 us, two tokens at 16 x 64K).
  static __device__ __forceinline__ void lone_nans(State& st, const Tile::Lanes& at, uint32_t vbase, int first, int loA, int LA,
                                                   int lo, int L) {
    constexpr int NB = kTokTile / kBlock;
    uint32_t any = 0;
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) any |= e4m3_nans(lds32(vbase + blk * kFp4BlockBytes + at.vs));
    if (!__any_sync(0xffffffffu, any)) return;
    uint32_t nan[2] = {0, 0};
#pragma unroll 1
    for (int blk = 0; blk < NB; ++blk) {
      const uint32_t addr = vbase + blk * kFp4BlockBytes + at.vs, sc = lds32(addr), bad = e4m3_nans(sc);
      const uint32_t a = fp4_visible_scales(bad, first + kBlock * blk, loA, LA);
      const uint32_t b = fp4_visible_scales(bad, first + kBlock * blk, lo, L);
      nan[0] |= a & ~b;
      nan[1] |= b & ~a;
      __syncwarp();   // lanes g and g ^ 1 hold the same scales: both have read them
      if (a ^ b) sts32(addr, sc & ~(a ^ b));
    }
    fence_proxy_async();   // before the next copy into this stage
    __syncwarp();
#pragma unroll
    for (int t = 0; t < 2; ++t) {   // the four lanes of g hold four tokens each of the same channels
      nan[t] |= __shfl_xor_sync(0xffffffffu, nan[t], 1);
      nan[t] |= __shfl_xor_sync(0xffffffffu, nan[t], 2);
      if (nan[t])
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) st.t[t].O[i][e] = __int_as_float(0x7fffffff);
    }
  }
  // EDGE as in TileState2::tile; V scales outside [loA, L) are cleared.
  template <bool EDGE>
  static __device__ __forceinline__ void tile(State& st, const Tile::Lanes& at, uint32_t kbase, uint32_t vbase, int tok0,
                                              int loA, int LA, int lo, int L, int lane) {
    constexpr int NB = kTokTile / kBlock;
    const int g = lane >> 2, c = lane & 3;
    if constexpr (EDGE) lone_nans(st, at, vbase, tok0 + 2 * c, loA, LA, lo, L);
    float s[2][NB][4];
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
      uint32_t a[4][4];
      fp4_k_fragments(kbase + blk * kFp4BlockBytes, at, a);
#pragma unroll
      for (int t = 0; t < 2; ++t) mma_f16_z(s[t][blk], a[0][0], a[0][1], a[0][2], a[0][3], st.t[t].q[0][0], st.t[t].q[0][1]);
#pragma unroll
      for (int k = 1; k < 4; ++k)
#pragma unroll
        for (int t = 0; t < 2; ++t)
          mma_f16(s[t][blk], a[k][0], a[k][1], a[k][2], a[k][3], st.t[t].q[k][0], st.t[t].q[k][1]);
    }
    if constexpr (EDGE) {
#pragma unroll
      for (int blk = 0; blk < NB; ++blk)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int tk = tok0 + kBlock * blk + g + 8 * e;
          if (tk < loA || tk >= LA) s[0][blk][2 * e] = s[0][blk][2 * e + 1] = -INFINITY;
          if (tk < lo || tk >= L) s[1][blk][2 * e] = s[1][blk][2 * e + 1] = -INFINITY;
        }
    }
    float2 neg[2], sum[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int blk = 0; blk < NB; ++blk) {
        mx[0] = max3(mx[0], s[t][blk][0], s[t][blk][2]);
        mx[1] = max3(mx[1], s[t][blk][1], s[t][blk][3]);
      }
      st.t[t].raise(mx);
      neg[t] = st.t[t].negated();
    }
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
      uint32_t b[2][2], a[4][4];
#pragma unroll
      for (int t = 0; t < 2; ++t) st.t[t].weights(s[t][blk], neg[t], blk == 0, sum[t], b[t][0], b[t][1]);
      fp4_v_fragments<EDGE>(vbase + blk * kFp4BlockBytes, at, tok0 + kBlock * blk + 2 * c, loA, L, a);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) mma_f16(st.t[t].O[i], a[i][0], a[i][1], a[i][2], a[i][3], b[t][0], b[t][1]);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) st.t[t].l_run = add2(st.t[t].l_run, sum[t]);
  }
};

}  // namespace
}  // namespace puzzle
