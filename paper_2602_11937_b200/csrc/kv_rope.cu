// Position rotation of the new tokens' queries and keys, fused with the quantise-and-append of keys and values into
// the paged cache (E4M3, bf16 or 4-bit codes; paper Section "KV Quantization": the cache is quantised as it is
// written).  Per row of 64 channels, with c and s the table's cosines and sines at the token's position:
//     out[i] = x[i] c[i] - x[j] s[i],   out[j] = x[j] c[i] + x[i] s[i]        (i, j) = (i, i + r/2) or (2i, 2i + 1)
// each product and the sum rounded to float32 (no contraction, so that the bytes are defined to the last bit), then
// q to bf16 and k, v to the cache's type as in kv_append.cu.  Reading and writing every byte once is all there is to
// do: a chunk is bound by HBM, a decode step by the chain of dependent loads (length -> table row, block -> store).
// Measured: 16 x 2048 tokens with 64 query and 8 KV heads 103 us into a bf16 cache (6.6 TB/s of read and written bytes),
// 102 E4M3 (6.3), 111 4-bit (5.7: sixteen-channel maxima, corrected quotients, byte-wide scale stores); one token for 16
// sequences 2.2 us, for 64 into the 4-bit cache 3.4.  Fewer heads per warp re-read the table's rows: 4 heads 5 % slower.
//
// Eight lanes hold a row, eight adjacent channels each: 16-byte loads, the rotation partner of the half-split form is
// one shuffle of packed pairs away, a 4-bit group is two lanes.
//  * chunk kernel: a warp takes four consecutive tokens and walks over eight heads, so that a token's cosines and sines
//    (256 bytes a row, twice the row itself) are fetched once for eight heads and eight loads are in flight; tokens are
//    aligned to four so that the two tokens that share V's bytes in a 4-bit block are in one warp.
//  * step kernel (one token per sequence): a group of eight lanes takes one (sequence, head), nothing is shared, the
//    launch is one chain of loads.
#include "common.cuh"
#include "decode_attn.cuh"
#include "kv_fp4.cuh"

namespace puzzle {
namespace {

enum Rotation { kNoRotation = 0, kHalves = 1, kAdjacent = 2 };

// Division by a head's scale, rounded as the IEEE quotient is: a power of two by its reciprocal, exactly; otherwise
// two Newton corrections of x * (1/s) with the correctly rounded reciprocal (Markstein, IBM J. Res. Dev. 34, 1990: the
// first leaves a quotient off by less than one ulp, the second rounds such a quotient correctly); scales outside
// [2^-60, 2^60] by the division itself.  Quotients below 2^-40 may lose their last bits, far below half the smallest
// code; beyond 2^100 they stay uncorrected, far above the largest.
struct Divisor {
  float s, r;
  int how;   // 0: power of two, 1: corrected reciprocal, 2: division
  __device__ __forceinline__ void set(float scale) {
    s = scale;
    const uint32_t bits = __float_as_uint(scale);
    const int e = (int)(bits >> 23) - 127;                        // negative scales: beyond 60
    how = (e < -60 || e > 60) ? 2 : ((bits & 0x7fffffu) == 0 ? 0 : 1);
    r = how == 2 ? 0.f : __frcp_rn(scale);
  }
  __device__ __forceinline__ void divide(float (&x)[8]) const {
    if (how == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= r;
    } else if (how == 1) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float q0 = x[i] * r;
        const float q1 = fmaf(fmaf(-q0, s, x[i]), r, q0);
        const float q2 = fmaf(fmaf(-q1, s, x[i]), r, q1);
        x[i] = fabsf(q0) < 0x1p100f ? copysignf(q2, x[i]) : q0;   // a NaN takes q0, which is it
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __fdiv_rn(x[i], s);
    }
  }
};

__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(f32x2_to_bf16x2(x[0], x[1]), f32x2_to_bf16x2(x[2], x[3]), f32x2_to_bf16x2(x[4], x[5]),
                    f32x2_to_bf16x2(x[6], x[7]));
}

// A lane's share of one position's table row, and the lane that holds its channels' partners.
template <int ROT>
struct Turn {
  float c[8], s[8];   // per channel, the sign of the sine's term included
  int partner;        // half-split form: lane of the partners
  bool turns;         // this lane's channels are rotated at all

  __device__ __forceinline__ void load(const float* row, int rotary, int lane) {
    const int o = lane & 7, half = rotary / 2;
    turns = 8 * o < rotary;
    partner = lane;
    if constexpr (ROT == kHalves) {
      const bool second = 8 * o >= half;
      if (turns) {
        partner = second ? lane - half / 8 : lane + half / 8;
        const float4* p = reinterpret_cast<const float4*>(row + 8 * o - (second ? half : 0));
        const float4* z = reinterpret_cast<const float4*>(row + half + 8 * o - (second ? half : 0));
        const float4 c0 = __ldg(p), c1 = __ldg(p + 1), s0 = __ldg(z), s1 = __ldg(z + 1);
        const float f = second ? 1.f : -1.f;
        c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
        s[0] = f * s0.x; s[1] = f * s0.y; s[2] = f * s0.z; s[3] = f * s0.w;
        s[4] = f * s1.x; s[5] = f * s1.y; s[6] = f * s1.z; s[7] = f * s1.w;
      }
    } else if constexpr (ROT == kAdjacent) {
      if (turns) {
        const float4 c0 = __ldg(reinterpret_cast<const float4*>(row + 4 * o));
        const float4 s0 = __ldg(reinterpret_cast<const float4*>(row + half + 4 * o));
        c[0] = c[1] = c0.x; c[2] = c[3] = c0.y; c[4] = c[5] = c0.z; c[6] = c[7] = c0.w;
        s[1] = s0.x; s[3] = s0.y; s[5] = s0.z; s[7] = s0.w;
#pragma unroll
        for (int i = 0; i < 8; i += 2) s[i] = -s[i + 1];
      }
    }
  }
  // x (the lane's channels, as loaded) -> rotated float32.  All lanes of the warp call it.
  __device__ __forceinline__ void apply(const uint4& raw, float (&x)[8]) const {
    unpack8(raw, x);
    if constexpr (ROT == kNoRotation) return;
    float y[8];
    if constexpr (ROT == kHalves) {
      uint4 other;
      other.x = __shfl_sync(0xffffffffu, raw.x, partner);
      other.y = __shfl_sync(0xffffffffu, raw.y, partner);
      other.z = __shfl_sync(0xffffffffu, raw.z, partner);
      other.w = __shfl_sync(0xffffffffu, raw.w, partner);
      unpack8(other, y);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
    }
    if (turns) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __fadd_rn(__fmul_rn(x[i], c[i]), __fmul_rn(y[i], s[i]));
    }
  }
};

// E4M3 codes of eight quotients; every NaN becomes the one canonical NaN code, as in kv_append.cu.
__device__ __forceinline__ uint2 encode8_e4m3(const float (&y)[8]) {
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c[i] = f32x2_to_e4m3x2(y[2 * i], y[2 * i + 1]);
    if (y[2 * i] != y[2 * i]) c[i] = (c[i] & 0xff00u) | 0x7fu;
    if (y[2 * i + 1] != y[2 * i + 1]) c[i] = (c[i] & 0x00ffu) | 0x7f00u;
  }
  return make_uint2((c[0] & 0xffffu) | (c[1] << 16), (c[2] & 0xffffu) | (c[3] << 16));
}

// Where a sequence's new tokens go.  `first` is the position of the first one (negative positions are skipped).
struct Span {
  int first, count;
  bool ok;
};
__device__ __forceinline__ Span span_of(const AppendParams& P, int b, bool reporter) {
  Span sp;
  const int len = P.seq_lens[b];
  sp.count = P.new_lens ? min(max(P.new_lens[b], 0), P.n_new) : P.n_new;
  sp.first = len - sp.count;
  sp.ok = len > 0 && sp.count > 0;
  if (len > P.max_blocks_per_seq * kBlock) {
    if (P.dev_status && reporter) atomicOr(P.dev_status, (int)PUZZLE_DEV_SEQ_TOO_LONG);
    sp.ok = false;
  }
  return sp;
}

// The table row of position `pos` of sequence b, or null (flagged) when the table has none.
__device__ __forceinline__ const float* table_row(const AppendParams& P, int b, int pos, bool reporter) {
  const long long at = (long long)pos + (P.pos_offset ? P.pos_offset[b] : 0);
  if (at < 0 || at >= P.num_positions) {
    if (P.dev_status && reporter) atomicOr(P.dev_status, (int)PUZZLE_DEV_BAD_POSITION);
    return nullptr;
  }
  return P.cos_sin + at * P.rotary;
}

// Physical block of position `pos`, or -1 (flagged) when the table's entry is out of range.
__device__ __forceinline__ long long block_of(const AppendParams& P, int b, int pos, bool reporter) {
  const long long blk = P.block_table ? (long long)P.block_table[(size_t)b * P.max_blocks_per_seq + pos / kBlock]
                                      : (long long)b * P.max_blocks_per_seq + pos / kBlock;
  if (blk >= 0 && blk < P.num_blocks) return blk;
  if (P.dev_status && reporter) atomicOr(P.dev_status, (int)PUZZLE_DEV_BAD_BLOCK);
  return -1;
}

// Stores the lane's eight channels of one token.  All lanes of the warp call it; `on` says whether this one has a token.
// PAIRS: lane ^ 8 holds the token that shares V's bytes (position ^ 1, or nothing: pair_on).
template <int KV, bool IS_V, bool PAIRS>
__device__ __forceinline__ void store8(void* cache, long long row, int slot, int o, const uint4& raw, float (&x)[8],
                                       const Divisor& div, bool turned, bool on, bool pair_on) {
  if constexpr (KV == PUZZLE_KV_BF16) {
    if (on)
      reinterpret_cast<uint4*>(cache)[(row * kBlock + slot) * (kHeadDim / 8) + o] = turned ? pack8(x) : raw;
  } else if constexpr (KV == PUZZLE_KV_FP8_E4M3) {
    div.divide(x);
    if (on) reinterpret_cast<uint2*>(cache)[(row * kBlock + slot) * (kHeadDim / 8) + o] = encode8_e4m3(x);
  } else {
    div.divide(x);
    uint32_t sc;
    const uint32_t w = fp4_quantise8(x, sc);
    uint8_t* base = static_cast<uint8_t*>(cache) + row * kFp4BlockBytes;
    if constexpr (!IS_V) {
      if (on) {
        *reinterpret_cast<uint32_t*>(base + 32 * slot + 4 * o) = w;
        if ((o & 1) == 0) base[fp4_k_scale_at(slot, o >> 1)] = (uint8_t)sc;
      }
    } else {
      uint32_t* at = reinterpret_cast<uint32_t*>(base + fp4_v_code_at(slot, 8 * o));
      const int odd = slot & 1;
      if constexpr (PAIRS) {
        const uint32_t other = __shfl_xor_sync(0xffffffffu, w, 8);
        if (on && pair_on) {   // this token and its neighbour: each lane writes half of the eight bytes
          const uint32_t even_w = odd ? other : w, odd_w = odd ? w : other;
          at[odd] = fp4_spread(even_w >> (16 * odd)) | (fp4_spread(odd_w >> (16 * odd)) << 4);
        }
      }
      if (on && !(PAIRS && pair_on)) {   // alone: the neighbour's nibbles stay
        const uint2 old = *reinterpret_cast<const uint2*>(at);
        const uint32_t keep = odd ? 0x0f0f0f0fu : 0xf0f0f0f0u;
        uint2 now;
        now.x = (old.x & keep) | (fp4_spread(w) << (4 * odd));
        now.y = (old.y & keep) | (fp4_spread(w >> 16) << (4 * odd));
        *reinterpret_cast<uint2*>(at) = now;
      }
      if (on && (o & 1) == 0) base[fp4_v_scale_at(slot, o >> 1)] = (uint8_t)sc;
    }
  }
}

constexpr int kHeadsPerWarp = 8;

}  // namespace

// Four blocks of 64 registers per SM where the codes are computed (three of 80: 108.5 against 102.4 us into the E4M3 cache,
// 116 against 111 into the 4-bit one); the bf16 copy has its loads in flight with three (103.5 against 104.7).
template <int KV, int ROT>
__global__ void __launch_bounds__(256, KV == PUZZLE_KV_BF16 ? 3 : 4) kv_append_chunk_kernel(const AppendParams P) {
  grid_dependency_wait();   // no early release, for the reason given in kv_append_kernel
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, o = lane & 7;
  const int b = blockIdx.z;
  const int kv_jobs = (P.Hkv + kHeadsPerWarp - 1) / kHeadsPerWarp;
  // keys, then values, then the query heads: the last blocks of the launch are quick ones (4 % at 16 x 2048 tokens)
  int job = blockIdx.y;
  const bool is_q = job >= 2 * kv_jobs, is_v = !is_q && job >= kv_jobs;
  job -= is_q ? 2 * kv_jobs : (is_v ? kv_jobs : 0);
  const bool reporter = o == 0 && blockIdx.y == 0;

  const Span sp = span_of(P, b, reporter);
  if (!sp.ok) return;
  const int pos = (max(sp.first, 0) & ~3) + (blockIdx.x * 8 + warp) * 4 + (lane >> 3);
  const int tok = pos - sp.first;
  bool on = pos >= sp.first && tok < sp.count;
  if (!__any_sync(0xffffffffu, on)) return;
  Turn<ROT> turn;
  if constexpr (ROT != kNoRotation) {
    const float* row = on ? table_row(P, b, pos, reporter) : nullptr;
    on = row != nullptr;
    if (!is_v) turn.load(on ? row : P.cos_sin, P.rotary, lane);
  }
  const int h0 = job * kHeadsPerWarp, heads = min(kHeadsPerWarp, (is_q ? P.Hq : P.Hkv) - h0);
  const __nv_bfloat16* src = is_q ? P.q + b * P.q_seq_stride + tok * P.q_token_stride
                                  : (is_v ? P.v + b * P.v_seq_stride + tok * P.v_token_stride
                                          : P.k + b * P.k_seq_stride + tok * P.k_token_stride);
  const uint4* in = reinterpret_cast<const uint4*>(src + h0 * kHeadDim) + o;
  uint4 raw[kHeadsPerWarp];
#pragma unroll
  for (int j = 0; j < kHeadsPerWarp; ++j)
    raw[j] = on && j < heads ? __ldcs(in + j * (kHeadDim / 8)) : make_uint4(0, 0, 0, 0);
  if (is_q) {
    uint4* out = reinterpret_cast<uint4*>(P.q_out + (((long long)b * P.n_new + tok) * P.Hq + h0) * kHeadDim) + o;
#pragma unroll
    for (int j = 0; j < kHeadsPerWarp; ++j) {
      float x[8];
      turn.apply(raw[j], x);
      if (on && j < heads) out[j * (kHeadDim / 8)] = pack8(x);
    }
    return;
  }
  long long blk = 0;
  if (on) {
    blk = block_of(P, b, pos, o == 0 && !is_v && job == 0);
    on = blk >= 0;
  }
  const bool pair_on = __shfl_xor_sync(0xffffffffu, (int)on, 8) != 0;
  const int slot = pos & (kBlock - 1);
  if (is_v) {
#pragma unroll
    for (int j = 0; j < kHeadsPerWarp; ++j) {
      if (j >= heads) break;
      float x[8];
      unpack8(raw[j], x);
      Divisor div;
      div.set(KV != PUZZLE_KV_BF16 && P.v_scale ? P.v_scale[h0 + j] : 1.f);
      store8<KV, true, true>(P.v_cache, blk * P.Hkv + h0 + j, slot, o, raw[j], x, div, false, on, pair_on);
    }
  } else {
#pragma unroll
    for (int j = 0; j < kHeadsPerWarp; ++j) {
      if (j >= heads) break;
      float x[8];
      turn.apply(raw[j], x);
      Divisor div;
      div.set(KV != PUZZLE_KV_BF16 && P.k_scale ? P.k_scale[h0 + j] : 1.f);
      store8<KV, false, true>(P.k_cache, blk * P.Hkv + h0 + j, slot, o, raw[j], x, div, ROT != kNoRotation, on, pair_on);
    }
  }
}

// One token per sequence: rows (query heads, keys, values) of all sequences, eight lanes each.
template <int KV, int ROT>
__global__ void __launch_bounds__(128) kv_append_step_kernel(const AppendParams P) {
  const int lane = threadIdx.x & 31, o = lane & 7;
  const int per_seq = (P.q ? P.Hq : 0) + 2 * P.Hkv;
  const int r = (blockIdx.x * blockDim.x + threadIdx.x) >> 3;
  int b = r / per_seq;
  const int m = r - b * per_seq;
  bool on = b < P.batch;
  if (!on) b = 0;
  const int hq = P.q ? P.Hq : 0;
  const bool is_q = m < hq, is_v = m >= hq + P.Hkv;
  const int h = is_q ? m : (is_v ? m - hq - P.Hkv : m - hq);
  const bool reporter = o == 0 && m == 0;
  const __nv_bfloat16* src = is_q ? P.q + b * P.q_seq_stride : (is_v ? P.v + b * P.v_seq_stride : P.k + b * P.k_seq_stride);
  grid_dependency_wait();   // no early release, for the reason given in kv_append_kernel
  const uint4 raw = __ldcs(reinterpret_cast<const uint4*>(src + h * kHeadDim) + o);
  Divisor div;
  div.set(1.f);
  if (KV != PUZZLE_KV_BF16 && !is_q) {
    const float* sc = is_v ? P.v_scale : P.k_scale;
    if (sc) div.set(__ldg(sc + h));
  }
  Span sp = span_of(P, b, on && reporter);
  const int pos = sp.first;                       // of the one new token, when there is one
  on = on && sp.ok && pos >= 0;
  long long blk = 0;
  bool block_ok = true;
  if (on && !is_q) {
    blk = block_of(P, b, pos, o == 0 && m == hq);
    block_ok = blk >= 0;
  }
  Turn<ROT> turn;
  if constexpr (ROT != kNoRotation) {
    const float* row = on ? table_row(P, b, pos, reporter) : nullptr;
    on = row != nullptr;
    turn.load(on ? row : P.cos_sin, P.rotary, lane);
    if (is_v) turn.turns = false;
  }
  float x[8];
  turn.apply(raw, x);
  if (is_q) {
    if (on) reinterpret_cast<uint4*>(P.q_out + ((long long)b * P.Hq + h) * kHeadDim)[o] = pack8(x);
    on = false;
  }
  on = on && block_ok;
  const int slot = pos & (kBlock - 1);
  // a 4-bit group spans two lanes of one row, so rows of K and V may meet in a warp without sharing anything
  if constexpr (KV == PUZZLE_KV_FP4_E2M1) {
    float xv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) xv[i] = x[i];
    store8<KV, false, false>(P.k_cache, blk * P.Hkv + h, slot, o, raw, x, div, true, on && !is_v, false);
    store8<KV, true, false>(P.v_cache, blk * P.Hkv + h, slot, o, raw, xv, div, false, on && is_v, false);
  } else {
    store8<KV, false, false>(is_v ? P.v_cache : P.k_cache, blk * P.Hkv + h, slot, o, raw, x, div,
                             ROT != kNoRotation && !is_v, on, false);
  }
}

template <int KV, int ROT>
static cudaError_t launch_append_variant(const AppendParams& P, cudaStream_t s) {
  const int hq = P.q ? P.Hq : 0;
  if (P.n_new == 1) {
    const long long threads = (long long)P.batch * (hq + 2 * P.Hkv) * 8;
    return launch_dependent(kv_append_step_kernel<KV, ROT>, dim3((unsigned)((threads + 127) / 128)), dim3(128), 0, s, P);
  }
  const int jobs = (hq + kHeadsPerWarp - 1) / kHeadsPerWarp + 2 * ((P.Hkv + kHeadsPerWarp - 1) / kHeadsPerWarp);
  const dim3 grid((unsigned)((P.n_new + 3 + 31) / 32), (unsigned)jobs, (unsigned)P.batch);
  return launch_dependent(kv_append_chunk_kernel<KV, ROT>, grid, dim3(256), 0, s, P);
}

template <int KV>
static cudaError_t launch_append_kv(const AppendParams& P, bool rotate, bool adjacent, cudaStream_t s) {
  if constexpr (KV == PUZZLE_KV_FP4_E2M1)   // the other types' plain appends are kv_append.cu's
    if (!rotate) return launch_append_variant<KV, kNoRotation>(P, s);
  return adjacent ? launch_append_variant<KV, kAdjacent>(P, s) : launch_append_variant<KV, kHalves>(P, s);
}

cudaError_t launch_append(const AppendParams& P, int kv_dtype, bool rotate, bool adjacent, cudaStream_t s) {
  switch (kv_dtype) {
    case PUZZLE_KV_FP8_E4M3: return launch_append_kv<PUZZLE_KV_FP8_E4M3>(P, rotate, adjacent, s);
    case PUZZLE_KV_BF16: return launch_append_kv<PUZZLE_KV_BF16>(P, rotate, adjacent, s);
    default: return launch_append_kv<PUZZLE_KV_FP4_E2M1>(P, rotate, adjacent, s);
  }
}

}  // namespace puzzle
