// The per-tile arithmetic of the split-KV kernels over the 4-bit cache (format: kv_fp4.cuh).  Include inside a
// translation unit only (internal linkage).
//
//  * An E2M1 code times its E4M3 group scale is exact in f16, so K and V are exact MMA operands: one convert and one
//    f16 multiply per two values, and the per-head scales factor out of both products as they do for the E4M3 cache.
//  * Here it is the tokens (S = K Q^T) and the channels (O^T = V^T P^T) that sit on the 16 MMA rows and the eight query
//    heads of the group that sit on the eight columns, so no half of an MMA is idle: 32 per tile of 64 tokens, half of
//    what the other tile arithmetic (decode_tile.cuh, heads on rows) issues, and O takes 16 registers instead of 32.
//    With 0.56 bytes per value the instruction stream, not HBM, is the nearer limit, so that is what the layout serves.
//  * The softmax weights then have to change sides: a lane holds P[token g][heads 2c, 2c+1] and needs P[tokens 2c,
//    2c+1][head g].  As packed f16 pairs that is one 8x8 transpose (movmatrix) per eight tokens.
//  * P is rounded to f16 once: 2^-11 relative, an eighth of the bf16 output's own rounding and independent from key to
//    key.  A second term for the remainder, as the other caches have it, is 16 more MMAs a tile and what feeds them: 112 to
//    125 us at 16 x 64K, 152 to 190 for two tokens.  The sum takes the float32 weights, so the lse has their accuracy.
//  * The reference of the weights is decode_tile.cuh's: weights down to 2^-26 of the largest keep all eleven bits, those
//    below are off by 2^-37 of the largest at most.  One vote per tile says whether some lane sees a weight beyond 2^15 of
//    it; only then it is raised (a reduction over the lanes, accumulators rescaled).
//  * A block arrives as it lies in HBM; every shared-memory read of a tile (8 bytes per lane of K and
//    V, 2 and 4 of the scales) is conflict free because the format's order is the fragments' order.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "decode_attn.cuh"
#include "decode_tile.cuh"
#include "kv_fp4.cuh"

namespace puzzle {
namespace {

__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
  uint16_t v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// a * b with b's low (high) half on both sides: the half select is part of the multiply, not an instruction.
__device__ __forceinline__ uint32_t hmul2_lo(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<__half2*>(&a), __low2half2(*reinterpret_cast<__half2*>(&b)));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t hmul2_hi(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<__half2*>(&a), __high2half2(*reinterpret_cast<__half2*>(&b)));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// Two float32 operations in one instruction, and the largest of three in one.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t"
      "add.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// 8x8 transpose of 16-bit cells: lane l holds row l / 4, columns 2 (l % 4) and the next, before and after.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
  return r;
}
// Four rows of a 2-D tensor (any four; rows outside it arrive as zeros), one below the other, in one tiled TMA load.
// The map's box is one row; x * element size a multiple of 16 bytes.
__device__ __forceinline__ void tma_gather4(uint32_t dst, const void* tmap, int x, int r0, int r1, int r2, int r3,
                                            uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes [%0], "
      "[%1, {%2, %3, %4, %5, %6}], [%7];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(r0), "r"(r1), "r"(r2), "r"(r3), "r"(bar)
      : "memory");
}

struct Fp4Lanes {
  uint32_t k, ks, v, vs;   // offsets within a block
  __device__ __forceinline__ void init(int lane) {
    const int g = lane >> 2, c = lane & 3;
    k = 32 * g + 8 * c;                                   // token g (+ 256: g + 8), channels 16c .. 16c+15
    ks = kFp4CodeBytes + 16 * c + 2 * g;                  // the scales of those two tokens, side by side
    v = 256 * (g >> 2) + 32 * c + 8 * (g & 3);            // tokens 2c, 2c+1 (+ 128: 2c+8, 2c+9), channels 8g .. 8g+7
    vs = kFp4CodeBytes + 16 * (g >> 1) + 4 * c;           // the scales of those four tokens
  }
};

// The scales of a lane's four V tokens with those outside [lo, L) cleared: their codes may be anything, and so may
// their scales (the NaN code included).  t = first of the four tokens' block plus 2c.
__device__ __forceinline__ uint32_t fp4_visible_scales(uint32_t sc, int t, int lo, int L) {
  uint32_t keep = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int tk = t + (i & 1) + 8 * (i >> 1);
    if (tk >= lo && tk < L) keep |= 0xffu << (8 * i);
  }
  return sc & keep;
}

// The MMA operands of one block.  K rows: tokens g, g + 8; k-step s covers channels 16c + 4s .. 16c + 4s + 3 of every c.
__device__ __forceinline__ void fp4_k_fragments(uint32_t block, const Fp4Lanes& at, uint32_t (&a)[4][4]) {
  const uint2 k0 = lds64(block + at.k), k1 = lds64(block + at.k + 256);
  const uint32_t sc = e4m3x2_to_f16x2(lds16(block + at.ks));
  e2m1x8_to_f16x2x4(k0.x, a[0][0], a[0][2], a[1][0], a[1][2]);
  e2m1x8_to_f16x2x4(k0.y, a[2][0], a[2][2], a[3][0], a[3][2]);
  e2m1x8_to_f16x2x4(k1.x, a[0][1], a[0][3], a[1][1], a[1][3]);
  e2m1x8_to_f16x2x4(k1.y, a[2][1], a[2][3], a[3][1], a[3][3]);
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    a[s][0] = hmul2_lo(a[s][0], sc); a[s][2] = hmul2_lo(a[s][2], sc);
    a[s][1] = hmul2_hi(a[s][1], sc); a[s][3] = hmul2_hi(a[s][3], sc);
  }
}
// V^T rows of m-tile i: channels 8g + 2i (row g) and 8g + 2i + 1 (row g + 8); columns: the 16 tokens in order.
template <bool EDGE>
__device__ __forceinline__ void fp4_v_fragments(uint32_t block, const Fp4Lanes& at, int t, int lo, int L,
                                                uint32_t (&a)[4][4]) {
  const uint2 v0 = lds64(block + at.v), v1 = lds64(block + at.v + 128);
  uint32_t sc = lds32(block + at.vs);
  if constexpr (EDGE) sc = fp4_visible_scales(sc, t, lo, L);
  const uint32_t s0 = e4m3x2_to_f16x2(sc), s1 = e4m3x2_to_f16x2(sc >> 16);
  e2m1x8_to_f16x2x4(v0.x, a[0][0], a[0][1], a[1][0], a[1][1]);
  e2m1x8_to_f16x2x4(v0.y, a[2][0], a[2][1], a[3][0], a[3][1]);
  e2m1x8_to_f16x2x4(v1.x, a[0][2], a[0][3], a[1][2], a[1][3]);
  e2m1x8_to_f16x2x4(v1.y, a[2][2], a[2][3], a[3][2], a[3][3]);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i][0] = hmul2(a[i][0], s0); a[i][1] = hmul2(a[i][1], s0);
    a[i][2] = hmul2(a[i][2], s1); a[i][3] = hmul2(a[i][3], s1);
  }
}

// Running state of one warp over the tiles of one (sequence, KV head) for one query token: heads 2c and 2c + 1 are this
// lane's columns.  O[i]: channels 8g + 2i (first two) and 8g + 2i + 1 (last two) of those heads.
struct Fp4State {
  uint32_t q[4][2];
  float alpha[2], m_ref[2];
  float2 l_run;
  float O[4][4];

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int e = 0; e < 2; ++e) m_ref[e] = -INFINITY;
    l_run = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) O[i][0] = O[i][1] = O[i][2] = O[i][3] = 0.f;
  }
  // qrow: query head g of the group (64 bf16).  As for the other caches the row is scaled by a power of two into f16,
  // exactly; the logit scale of head g takes it back and moves to the lanes that hold the head's column.
  __device__ __forceinline__ void load_query(const __nv_bfloat16* qrow, float ks, float sm_scale_log2e, int lane) {
    const int c = lane & 3;
    float x[16];
    float amax = 0.f;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const uint2 raw = *reinterpret_cast<const uint2*>(qrow + 16 * c + 4 * s);
      x[4 * s] = __uint_as_float(raw.x << 16);
      x[4 * s + 1] = __uint_as_float(raw.x & 0xffff0000u);
      x[4 * s + 2] = __uint_as_float(raw.y << 16);
      x[4 * s + 3] = __uint_as_float(raw.y & 0xffff0000u);
#pragma unroll
      for (int i = 0; i < 4; ++i) amax = fmaxf(amax, fabsf(x[4 * s + i]));
    }
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    int shift = 0;
    if (amax > 0.f) {
      shift = -((int)(__float_as_uint(amax) >> 23) - 127);  // amax * 2^shift in [1, 2)
      shift = max(-120, min(120, shift));
    }
    const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
    const float down = __uint_as_float((uint32_t)(127 - shift) << 23);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      q[s][0] = f32x2_to_f16x2(x[4 * s] * up, x[4 * s + 1] * up);
      q[s][1] = f32x2_to_f16x2(x[4 * s + 2] * up, x[4 * s + 3] * up);
    }
    const float a = fmaxf(sm_scale_log2e * ks * down, 1e-30f);  // keeps (-inf) * alpha = -inf for masked keys
    alpha[0] = __shfl_sync(0xffffffffu, a, 8 * c);
    alpha[1] = __shfl_sync(0xffffffffu, a, 8 * c + 4);
  }
  // Raises the references where a head's logits (mx: this lane's largest, code units) exceed them by 2^kTopLog2.
  __device__ __forceinline__ void raise(float (&mx)[2]) {
    const float t0 = mx[0] * alpha[0], t1 = mx[1] * alpha[1];
    if (!__any_sync(0xffffffffu, t0 > m_ref[0] + kTopLog2 || t1 > m_ref[1] + kTopLog2)) return;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float m = e ? t1 : t0;
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
      if (m > m_ref[e] + kTopLog2) {
        m -= kRefLog2;
        const float corr = ex2(m_ref[e] - m);   // 0 on the first visible tile
        if (e) l_run.y *= corr; else l_run.x *= corr;
#pragma unroll
        for (int i = 0; i < 4; ++i) { O[i][e] *= corr; O[i][2 + e] *= corr; }
        m_ref[e] = m;
      }
    }
  }
  // Weights of one block's logits s[4] (token g: heads 2c, 2c+1; token g + 8) as the B operand of O^T += V^T P^T.  They are
  // added up over a tile's blocks before they join l_run, which rounds a long tail below one key a quarter as often.
  __device__ __forceinline__ void weights(const float (&s)[4], float2 neg, bool first, float2& sum, uint32_t& b0, uint32_t& b1) {
    const float2 al = make_float2(alpha[0], alpha[1]);
    const float2 t0 = fma2(make_float2(s[0], s[1]), al, neg), t1 = fma2(make_float2(s[2], s[3]), al, neg);
    const float2 p0 = make_float2(ex2(t0.x), ex2(t0.y)), p1 = make_float2(ex2(t1.x), ex2(t1.y));
    sum = first ? add2(p0, p1) : add2(sum, add2(p0, p1));
    b0 = transpose8x8(f32x2_to_f16x2(p0.x, p0.y));
    b1 = transpose8x8(f32x2_to_f16x2(p1.x, p1.y));
  }
  __device__ __forceinline__ float2 negated() const {
    return make_float2(m_ref[0] == -INFINITY ? 0.f : -m_ref[0], m_ref[1] == -INFINITY ? 0.f : -m_ref[1]);
  }
};

// The 4-bit cache as the split-KV kernels see it (see SwizzledTile in decode_tile.cuh).
struct Fp4Tile {
  static constexpr int kBlockBytes = kFp4BlockBytes;
  static constexpr bool kScaled = true;
  static constexpr int kAlign = 128;
  using Lanes = Fp4Lanes;
  using State = Fp4State;

  static __device__ __forceinline__ void prefetch(const DecodeParams& P) {
    tma_prefetch_desc(&P.tmK);
    tma_prefetch_desc(&P.tmV);
  }
  // One gather of four rows brings the K (V) blocks of 64 tokens, wherever they are: the tensor maps' rows are blocks.
  template <int NB>
  static __device__ __forceinline__ void load_tile(const DecodeParams& P, uint32_t stage, int row, uint32_t bar) {
    static_assert(NB % 4 == 0, "whole gathers");
    int rows[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) rows[i] = __shfl_sync(0xffffffffu, row, i);
    if (elect_one()) {
      mbar_arrive_expect_tx(bar, 2 * NB * kBlockBytes);
#pragma unroll
      for (int i = 0; i < NB; i += 4) {
        tma_gather4(stage + i * kBlockBytes, &P.tmK, 0, rows[i], rows[i + 1], rows[i + 2], rows[i + 3], bar);
        tma_gather4(stage + (NB + i) * kBlockBytes, &P.tmV, 0, rows[i], rows[i + 1], rows[i + 2], rows[i + 3], bar);
      }
    }
  }
  static __device__ __forceinline__ void load_query(State& st, const __nv_bfloat16* qrow, float ks, float sm, int lane) {
    st.load_query(qrow, ks, sm, lane);
  }
  template <int TT, bool EDGE>
  static __device__ __forceinline__ void tile(State& st, const Lanes& at, uint32_t kbase, uint32_t vbase, int tok0, int lo,
                                              int L, int lane) {
    constexpr int NB = TT / kBlock;
    const int g = lane >> 2, c = lane & 3;
    float s[NB][4];
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
      uint32_t a[4][4];
      fp4_k_fragments(kbase + blk * kFp4BlockBytes, at, a);
      mma_f16_z(s[blk], a[0][0], a[0][1], a[0][2], a[0][3], st.q[0][0], st.q[0][1]);
#pragma unroll
      for (int k = 1; k < 4; ++k) mma_f16(s[blk], a[k][0], a[k][1], a[k][2], a[k][3], st.q[k][0], st.q[k][1]);
    }
    if constexpr (EDGE) {
#pragma unroll
      for (int blk = 0; blk < NB; ++blk)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int tk = tok0 + kBlock * blk + g + 8 * e;
          if (tk < lo || tk >= L) s[blk][2 * e] = s[blk][2 * e + 1] = -INFINITY;
        }
    }
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
      mx[0] = max3(mx[0], s[blk][0], s[blk][2]);
      mx[1] = max3(mx[1], s[blk][1], s[blk][3]);
    }
    st.raise(mx);
    const float2 neg = st.negated();
    float2 sum;
#pragma unroll
    for (int blk = 0; blk < NB; ++blk) {
      uint32_t b0, b1, a[4][4];
      st.weights(s[blk], neg, blk == 0, sum, b0, b1);
      fp4_v_fragments<EDGE>(vbase + blk * kFp4BlockBytes, at, tok0 + kBlock * blk + 2 * c, lo, L, a);
#pragma unroll
      for (int i = 0; i < 4; ++i) mma_f16(st.O[i], a[i][0], a[i][1], a[i][2], a[i][3], b0, b1);
    }
    st.l_run = add2(st.l_run, sum);
  }
  // The state of head g on the four lanes of g, as the kernels combine and store it: lane c of the four gets channels
  // 16c + j in o[j][0] and 16c + 8 + j in o[j][1].
  static __device__ __forceinline__ void finish(const State& st, float& m, float& l, float (&o)[8][2], int lane) {
    const int g = lane >> 2;
    float l0 = st.l_run.x, l1 = st.l_run.y;
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
      l0 += __shfl_xor_sync(0xffffffffu, l0, d);
      l1 += __shfl_xor_sync(0xffffffffu, l1, d);
    }
    // head g's column pair is held by lanes with c = g / 2
    const float ma = __shfl_sync(0xffffffffu, st.m_ref[0], g >> 1), mb = __shfl_sync(0xffffffffu, st.m_ref[1], g >> 1);
    const float la = __shfl_sync(0xffffffffu, l0, g >> 1), lb = __shfl_sync(0xffffffffu, l1, g >> 1);
    m = (g & 1) ? mb : ma;
    l = (g & 1) ? lb : la;
    if (!(l >= 0.f)) {   // a NaN among the weights: nothing downstream may take this for an empty part
      l = INFINITY;
      if (m == -INFINITY) m = 0.f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {   // float32 8x8 transposes, as two 16-bit ones
      const uint32_t x = __float_as_uint(st.O[j >> 1][2 * (j & 1)]), y = __float_as_uint(st.O[j >> 1][2 * (j & 1) + 1]);
      const uint32_t low = transpose8x8(prmt(x, y, 0x5410u)), high = transpose8x8(prmt(x, y, 0x7632u));
      o[j][0] = __uint_as_float(prmt(low, high, 0x5410u));
      o[j][1] = __uint_as_float(prmt(low, high, 0x7632u));
    }
  }
  static __device__ __forceinline__ void store(float* row, const float (&o)[8][2], float f, int c) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int j = 0; j < 8; j += 4)
        *reinterpret_cast<float4*>(row + 16 * c + 8 * e + j) =
            make_float4(o[j][e] * f, o[j + 1][e] * f, o[j + 2][e] * f, o[j + 3][e] * f);
  }
  static __device__ __forceinline__ void store(__nv_bfloat16* row, const float (&o)[8][2], float f, int c) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
      *reinterpret_cast<uint4*>(row + 16 * c + 8 * e) =
          make_uint4(f32x2_to_bf16x2(o[0][e] * f, o[1][e] * f), f32x2_to_bf16x2(o[2][e] * f, o[3][e] * f),
                     f32x2_to_bf16x2(o[4][e] * f, o[5][e] * f), f32x2_to_bf16x2(o[6][e] * f, o[7][e] * f));
  }
};

}  // namespace
}  // namespace puzzle
