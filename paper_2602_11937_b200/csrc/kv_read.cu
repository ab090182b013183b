// Cached tokens back as bf16: the last read_lens[b] tokens of every sequence, dequantised with the head's scale (and
// the 4-bit group's).  What a consumer of contiguous K/V needs (the attention of a prompt chunk over its own rounded
// keys and values, a cache handed to another worker) and the only way to look into a 4-bit block short of decoding its
// layout.  HBM-bound: 0.56 to 2 bytes read and 2 written per value.
//
// Measured, 16 x 8192 tokens: 59 us from a 4-bit cache (5.8 TB/s of read and written bytes), 67 E4M3 (6.1), 82 bf16 (6.5).
// Eight lanes hold a row (one token of one head), eight channels each; a warp takes four consecutive tokens and walks
// over eight heads with all loads in flight, so the 1 KiB a token occupies in the output is written by one warp.
#include "common.cuh"
#include "decode_attn.cuh"
#include "kv_fp4.cuh"

namespace puzzle {
namespace {
constexpr int kReadHeads = 8;
}

template <int KV>
__global__ void __launch_bounds__(256) kv_read_tokens_kernel(const ReadParams P) {
  grid_dependency_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, o = lane & 7;
  const int b = blockIdx.z, jobs = (P.Hkv + kReadHeads - 1) / kReadHeads;
  const bool is_v = blockIdx.y >= jobs;
  const int h0 = (blockIdx.y - (is_v ? jobs : 0)) * kReadHeads, heads = min(kReadHeads, P.Hkv - h0);
  const int len = P.seq_lens[b];
  const int count = P.read_lens ? min(max(P.read_lens[b], 0), P.n_read) : P.n_read;
  if (len > P.max_blocks_per_seq * kBlock) {
    if (P.dev_status && threadIdx.x == 0 && blockIdx.x == 0 && blockIdx.y == 0)
      atomicOr(P.dev_status, (int)PUZZLE_DEV_SEQ_TOO_LONG);
    return;
  }
  const int tok = (blockIdx.x * 8 + warp) * 4 + (lane >> 3);
  const int pos = len - count + tok;
  if (tok >= count || pos < 0) return;   // no shuffles below
  const long long blk = P.block_table ? (long long)P.block_table[(size_t)b * P.max_blocks_per_seq + pos / kBlock]
                                      : (long long)b * P.max_blocks_per_seq + pos / kBlock;
  const bool ok = blk >= 0 && blk < P.num_blocks;
  if (!ok && P.dev_status && o == 0) atomicOr(P.dev_status, (int)PUZZLE_DEV_BAD_BLOCK);
  const int slot = pos & (kBlock - 1);
  const void* cache = is_v ? P.v_cache : P.k_cache;
  const float* scales = is_v ? P.v_scale : P.k_scale;
  uint4* out = reinterpret_cast<uint4*>((is_v ? P.v_out : P.k_out) +
                                        (((long long)b * P.n_read + tok) * P.Hkv + h0) * kHeadDim) + o;
  const long long row = blk * P.Hkv + h0;
  uint4 raw[kReadHeads];
  uint32_t sc[kReadHeads];
#pragma unroll
  for (int j = 0; j < kReadHeads; ++j) {
    raw[j] = make_uint4(0, 0, 0, 0);
    sc[j] = 0;
    if (!ok || j >= heads) continue;
    if constexpr (KV == PUZZLE_KV_BF16) {
      raw[j] = __ldcs(reinterpret_cast<const uint4*>(cache) + ((row + j) * kBlock + slot) * (kHeadDim / 8) + o);
    } else if constexpr (KV == PUZZLE_KV_FP8_E4M3) {
      const uint2 v = __ldcs(reinterpret_cast<const uint2*>(cache) + ((row + j) * kBlock + slot) * (kHeadDim / 8) + o);
      raw[j].x = v.x; raw[j].y = v.y;
    } else {
      const uint8_t* base = static_cast<const uint8_t*>(cache) + (row + j) * kFp4BlockBytes;
      if (is_v) {
        const uint2 v = *reinterpret_cast<const uint2*>(base + fp4_v_code_at(slot, 8 * o));
        raw[j].x = v.x; raw[j].y = v.y;
        sc[j] = base[fp4_v_scale_at(slot, o >> 1)];
      } else {
        raw[j].x = *reinterpret_cast<const uint32_t*>(base + 32 * slot + 4 * o);
        sc[j] = base[fp4_k_scale_at(slot, o >> 1)];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kReadHeads; ++j) {
    if (j >= heads) break;
    uint4 v = raw[j];
    if constexpr (KV != PUZZLE_KV_BF16) {
      const float s = scales ? __ldg(scales + h0 + j) : 1.f;
      uint32_t h[4];   // eight f16 values
      float t = 1.f;
      if constexpr (KV == PUZZLE_KV_FP8_E4M3) {
        h[0] = e4m3x2_to_f16x2(v.x); h[1] = e4m3x2_to_f16x2(v.x >> 16);
        h[2] = e4m3x2_to_f16x2(v.y); h[3] = e4m3x2_to_f16x2(v.y >> 16);
      } else {
        uint32_t w = v.x;
        if (is_v) {
          const int sh = 4 * (slot & 1);
          w = fp4_gather(v.x >> sh) | (fp4_gather(v.y >> sh) << 16);
        }
        e2m1x8_to_f16x2x4(w, h[0], h[1], h[2], h[3]);
        t = f16_lo_to_f32(e4m3x2_to_f16x2(sc[j]));
      }
      float x[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {   // code * t is exact, so this is one rounding to float32 and one to bf16
        x[2 * i] = f16_lo_to_f32(h[i]) * t * s;
        x[2 * i + 1] = f16_hi_to_f32(h[i]) * t * s;
      }
      v = make_uint4(f32x2_to_bf16x2(x[0], x[1]), f32x2_to_bf16x2(x[2], x[3]), f32x2_to_bf16x2(x[4], x[5]),
                     f32x2_to_bf16x2(x[6], x[7]));
    }
    __stcs(out + j * (kHeadDim / 8), v);
  }
}

cudaError_t launch_read_tokens(const ReadParams& P, int kv_dtype, cudaStream_t s) {
  const dim3 grid((unsigned)((P.n_read + 31) / 32), (unsigned)(2 * ((P.Hkv + kReadHeads - 1) / kReadHeads)),
                  (unsigned)P.batch);
  switch (kv_dtype) {
    case PUZZLE_KV_FP8_E4M3:
      return launch_dependent(kv_read_tokens_kernel<PUZZLE_KV_FP8_E4M3>, grid, dim3(256), 0, s, P);
    case PUZZLE_KV_BF16: return launch_dependent(kv_read_tokens_kernel<PUZZLE_KV_BF16>, grid, dim3(256), 0, s, P);
    default: return launch_dependent(kv_read_tokens_kernel<PUZZLE_KV_FP4_E2M1>, grid, dim3(256), 0, s, P);
  }
}

}  // namespace puzzle
