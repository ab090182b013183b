// The 4-bit cache format: E2M1 codes with one E4M3 scale per 16 channels of a token, on top of the per-head float32
// scale that the E4M3 cache has too.  With y = x / scale[h]:
//     t = E4M3(max |y| / 6) over the 16 channels,   code = E2M1(y / t),   x ~ code * t * scale[h]
// (6 is the largest E2M1 value, so the largest channel of a group lands on it).  A group with a NaN keeps it: its
// scale is the NaN code.  The product code * t has at most six significant bits and lies between 2^-10 and 2688, so it
// is exact in f16 and in bf16; that is what lets the attention kernels feed it to f16 MMAs without any rounding.
//
// One (block, KV head) is 576 bytes: 512 bytes of codes, then 64 scales.  The order of both is the order in which a
// warp's MMA fragments want them (decode_tile_fp4.cuh), so that every shared-memory read of a tile is conflict free and
// needs no rearrangement:
//     K codes   token t at bytes 32 t ..; channel d in byte d / 2, the even channel in the low nibble
//     V codes   byte 256 (d / 32) + 32 (t / 2) + d % 32, the even token in the low nibble: P.V contracts over tokens,
//               so the two tokens of an f16 pair have to come out of one byte
//     scales    16 b + 2 (t % 8) + t / 8 (K) and 16 b + 4 ((t % 8) / 2) + 2 (t / 8) + t % 2 (V), b = d / 16
// Because two tokens share V's bytes, writing one of them keeps the other's nibbles.
#pragma once

#include "common.cuh"

namespace puzzle {
namespace {

constexpr int kFp4Group = 16;                    // channels that share an E4M3 scale
constexpr int kFp4CodeBytes = kBlock * kHeadDim / 2;
constexpr int kFp4BlockBytes = PUZZLE_FP4_BLOCK_BYTES;
static_assert(kFp4BlockBytes == kFp4CodeBytes + kBlock * kHeadDim / kFp4Group, "codes, then scales");

__device__ __forceinline__ int fp4_k_scale_at(int t, int b) { return kFp4CodeBytes + 16 * b + 2 * (t & 7) + (t >> 3); }
__device__ __forceinline__ int fp4_v_scale_at(int t, int b) {
  return kFp4CodeBytes + 16 * b + 4 * ((t & 7) >> 1) + 2 * (t >> 3) + (t & 1);
}
__device__ __forceinline__ int fp4_v_code_at(int t, int d) { return 256 * (d >> 5) + 32 * (t >> 1) + (d & 31); }

// Two floats -> two E2M1 codes (nearest, ties to even, saturating at 6); `lo` in the low nibble.
__device__ __forceinline__ uint32_t f32x2_to_e2m1x2(float lo, float hi) {
  uint32_t r;
  asm("{\n\t.reg .b8 c;\n\tcvt.rn.satfinite.e2m1x2.f32 c, %1, %2;\n\tcvt.u32.u8 %0, c;\n\t}" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// The four bytes of `r`, each two E2M1 codes, as four f16 pairs (low nibble in the low half).
__device__ __forceinline__ void e2m1x8_to_f16x2x4(uint32_t r, uint32_t& h0, uint32_t& h1, uint32_t& h2, uint32_t& h3) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h0), "=r"(h1), "=r"(h2), "=r"(h3)
      : "r"(r));
}
// Two E4M3 codes -> two f16 values (exact).
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t codes) {
  uint32_t r;
  asm("{\n\t.reg .b16 c;\n\tcvt.u16.u32 c, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, c;\n\t}" : "=r"(r) : "r"(codes));
  return r;
}
__device__ __forceinline__ float f16_lo_to_f32(uint32_t h) {
  float f;
  asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %1;\n\tcvt.f32.f16 %0, l;\n\t}" : "=f"(f) : "r"(h));
  return f;
}
__device__ __forceinline__ float f16_hi_to_f32(uint32_t h) {
  float f;
  asm("{\n\t.reg .b16 l, u;\n\tmov.b32 {l, u}, %1;\n\tcvt.f32.f16 %0, u;\n\t}" : "=f"(f) : "r"(h));
  return f;
}

// Quantises the eight channels a lane holds (y already divided by the head's scale); the neighbouring lane (lane ^ 1)
// holds the other half of the group.  Returns the eight codes (channel i in nibble i) and the group's scale code.
__device__ __forceinline__ uint32_t fp4_quantise8(float (&y)[8], uint32_t& scale_code) {
  uint32_t top = 0;   // as integers: NaN above infinity above every number
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(y[i]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  const float a = __uint_as_float(top);
  const bool nan = top > 0x7f800000u;
  scale_code = nan ? 0x7fu : (f32x2_to_e4m3x2(__fdiv_rn(a, 6.f), 0.f) & 0xffu);
  const float t = f16_lo_to_f32(e4m3x2_to_f16x2(scale_code));
  const bool none = nan || scale_code == 0;
  const float r = none ? 0.f : __frcp_rn(t);
  if (a > 4096.f)   // codes saturate long before; keeps infinities out of the correction below
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(y[i], -8192.f), 8192.f);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    // y / t with one Newton correction (Markstein, IBM J. Res. Dev. 34, 1990): at most a hair over half an ulp off.
    // y and t * border are both float32, and t has four significant bits, so y / t is either exactly a border between
    // two codes (then the corrected quotient is exact) or further from it than that: the code is the nearest one.
    float q[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float q0 = y[i + e] * r;
      q[e] = none ? 0.f : copysignf(fmaf(fmaf(-q0, t, y[i + e]), r, q0), y[i + e]);
    }
    w |= f32x2_to_e2m1x2(q[0], q[1]) << (4 * i);
  }
  return w;
}

// Nibbles 0..3 of x -> the low nibbles of four bytes.
__device__ __forceinline__ uint32_t fp4_spread(uint32_t x) {
  x &= 0xffffu;
  x = (x | (x << 8)) & 0x00ff00ffu;
  return (x | (x << 4)) & 0x0f0f0f0fu;
}
// The low nibbles of four bytes -> 16 bits.
__device__ __forceinline__ uint32_t fp4_gather(uint32_t x) {
  x &= 0x0f0f0f0fu;
  x = (x | (x >> 4)) & 0x00ff00ffu;
  return (x | (x >> 8)) & 0xffffu;
}

}  // namespace
}  // namespace puzzle
