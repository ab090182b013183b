// Decode attention over the 4-bit cache for launches that need no cutting: a group of GW warps takes a (sequence, KV head)
// pair whole, warp i of the group its tiles i, i + GW, ..., and the warps' states meet in shared memory.
//
// Cut evenly over all warps of the chip, a short or middling launch has almost as many partials as tiles, and merging
// them through L2 is a chain of dependent trips that grows with their number; handing tiles out inside a CTA
// (decode_attn_cta.cu) costs a claim and a record per tile, which weighs on 4-bit tiles (half the bytes of an E4M3 tile,
// as many instructions).  Here no schedule is built, nothing is claimed, nothing but inputs and outputs touches
// global memory, and a pair's end is one barrier of its group and one output value per thread (GW = 16).  Sixteen warps
// per CTA: the tile loop needs 119 registers without spilling.  What limits it is balance: the launch lasts as long as the SM
// with the most tiles, which is why the host takes it only when the pairs fill the SMs evenly enough or the launch is
// short (pick_kernel in api.cu).  Measured, group / next best kernel, us: 4 x 1024 tokens 6.2 / 13.9, 16 x 4096 11.8 /
// 20.2, 16 x 16384 34.8 / 44, 64 x 4096 33.8 / 41, 256 x 1024 33.6 / 44.5, 256 x 4096 110 / 122.
#include <cuda.h>

#include <climits>

#include "common.cuh"
#include "decode_attn.cuh"
#include "decode_tile.cuh"
#include "decode_tile_fp4.cuh"

namespace puzzle {
namespace {

constexpr int kGrpWarps = 16, kGrpStages = 2, kGrpTile = 64;

template <int GW>
__device__ __forceinline__ void group_sync(int group) {
  if constexpr (GW == 1) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(GW * 32) : "memory");
}

}  // namespace

template <int GW, typename F>
__global__ void __launch_bounds__(kGrpWarps * 32, 1) decode_attn_group_kernel(const __grid_constant__ DecodeParams P) {
  constexpr int NW = kGrpWarps, NS = kGrpStages, TT = kGrpTile, NB = TT / kBlock, NG = NW / GW;
  constexpr int STAGE_BYTES = 2 * NB * F::kBlockBytes;
  constexpr int VEC = kGroup * kHeadDim / (GW * 32);   // output values per thread when a pair is combined
  static_assert(NW % GW == 0, "whole groups");
  static_assert(NS == 2, "the other stage is stage ^ 1");

  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  uint8_t* sp = smem_raw + (((raw + F::kAlign - 1u) & ~(F::kAlign - 1u)) - raw);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, c = lane & 3;
  const int group = warp / GW, wi = warp % GW;
  const uint32_t pipe = smem_u32(sp) + warp * (NS * STAGE_BYTES);   sp += NW * NS * STAGE_BYTES;
  float* dep_o = reinterpret_cast<float*>(sp);                      sp += NW * kGroup * kHeadDim * sizeof(float);  // [warp][head][channel]
  float* dep_m = reinterpret_cast<float*>(sp);                      sp += NW * kGroup * sizeof(float);             // [warp][head]
  float* dep_l = reinterpret_cast<float*>(sp);                      sp += NW * kGroup * sizeof(float);
  const uint32_t bars = smem_u32(sp) + warp * (NS * 8);
  dep_o += group * GW * kGroup * kHeadDim;
  dep_m += group * GW * kGroup;
  dep_l += group * GW * kGroup;

  if (lane == 0) {
#pragma unroll
    for (int i = 0; i < NS; ++i) mbar_init(bars + 8 * i, 1);
    fence_mbar_init();
  }
  if (threadIdx.x == 0) F::prefetch(P);
  release_dependents();
  grid_dependency_wait();   // nothing above reads or writes global memory
  __syncwarp();

  typename F::Lanes at;
  at.init(lane);
  const int pairs = P.batch * P.Hkv, step = gridDim.x * NG;

  // ---- the pair whose tiles are issued and computed, and this warp's copies: two tiles ahead, table entries three
  int b, kvh, t_end;
  SeqRange r;
  int t_issue, phys;     // next tile to issue, and its blocks (lane i < NB: block i)
  int stage = 0;
  uint32_t phase = 0;
  bool failed = false;   // a copy did not land in time: this warp stops computing but keeps in step with its group
  auto lookup = [&]() {
    phys = INT_MIN;
    const int j = t_issue * NB + lane;
    if (t_issue < t_end && lane < NB && j * kBlock < r.L && j * kBlock + kBlock > r.lo)
      phys = P.block_table ? P.block_table[(size_t)b * P.max_blocks_per_seq + j] : b * P.max_blocks_per_seq + j;
  };
  auto issue = [&](int st) {
    if (t_issue >= t_end) return;
    int row = P.oob_row;
    if (lane < NB) {
      if (phys >= 0 && phys < P.num_blocks) row = (phys * P.Hkv + kvh) * P.rows_per_block;
      else if (phys != INT_MIN && P.dev_status) atomicOr(P.dev_status, (int)PUZZLE_DEV_BAD_BLOCK);
    }
    F::template load_tile<NB>(P, pipe + st * STAGE_BYTES, row, bars + 8 * st, lane, [] {});
    t_issue += GW;
    lookup();
  };
  auto start = [&](int p) {   // the pair and its first copies; all earlier tiles of this warp have been consumed
    b = p / P.Hkv;
    kvh = p - b * P.Hkv;
    bool too_long;
    r = seq_range(P.seq_lens[b], P.window, P.max_blocks_per_seq * kBlock, TT, too_long);
    if (too_long && P.dev_status && kvh == 0 && wi == 0 && lane == 0)
      atomicOr(P.dev_status, (int)PUZZLE_DEV_SEQ_TOO_LONG);
    t_end = r.tlo + r.ntile;
    t_issue = failed ? t_end : r.tlo + wi;
    lookup();
#pragma unroll
    for (int i = 0; i < NS; ++i) issue((stage + i) % NS);
  };

  int p = group * gridDim.x + blockIdx.x;   // neighbouring pairs on different SMs
  if (p < pairs) start(p);
#pragma unroll 1
  while (p < pairs) {
    typename F::State st;
    st.reset();
    if (r.tlo + wi < t_end)
      F::load_query(st, P.q + ((size_t)b * (P.Hkv * kGroup) + kvh * kGroup + g) * kHeadDim,
                    P.k_scale && F::kScaled ? P.k_scale[kvh] : 1.f, P.sm_scale_log2e, lane);
#pragma unroll 1
    for (int t = r.tlo + wi; t < t_end && !failed; t += GW) {
      if (!mbar_wait_bounded(bars + 8 * stage, phase)) {
        if (P.dev_status && lane == 0) atomicOr(P.dev_status, (int)PUZZLE_DEV_WAIT_EXPIRED);
        failed = true;
        // the other copy in flight gets a bounded chance to land: nothing of this warp is under way when it goes on
        if (t + GW < t_issue) mbar_wait_bounded(bars + 8 * (stage ^ 1), phase ^ (uint32_t)stage);
        break;
      }
      const uint32_t kbase = pipe + stage * STAGE_BYTES, vbase = kbase + NB * F::kBlockBytes;
      const int tok0 = t * TT;
      if (tok0 < r.lo || tok0 + TT > r.L) F::template tile<TT, true>(st, at, kbase, vbase, tok0, r.lo, r.L, lane);
      else F::template tile<TT, false>(st, at, kbase, vbase, tok0, r.lo, r.L, lane);
      __syncwarp();
      issue(stage);
      if (++stage == NS) { stage = 0; phase ^= 1u; }
    }
    const int b_done = b, kvh_done = kvh, parts = min(r.ntile, GW);
    p += step;
    if (p < pairs) start(p);   // the next pair's first tiles are on their way while this one is combined

    // ---- the warps' states meet; one without a tile leaves an empty one
    float m, l, o[8][2];
    F::finish(st, m, l, o, lane);
    F::store(dep_o + (wi * kGroup + g) * kHeadDim, o, 1.f, c);
    if (c == 0) {
      dep_m[wi * kGroup + g] = l == 0.f ? -INFINITY : m;
      dep_l[wi * kGroup + g] = l;
    }
    group_sync<GW>(group);
    const int e = (wi * 32 + lane) * VEC, h = e / kHeadDim, d = e % kHeadDim;
    const int head = kvh_done * kGroup + h;
    const float sink = P.sinks ? P.sinks[head] * 1.4426950408889634f : -INFINITY;
    float M = sink, Z = 0.f, acc[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
    for (int u = 0; u < parts; ++u) M = fmaxf(M, dep_m[u * kGroup + h]);
    if (M != -INFINITY) {
      Z = sink == -INFINITY ? 0.f : ex2(sink - M);
      for (int u = 0; u < parts; ++u) {
        const float f = ex2(dep_m[u * kGroup + h] - M);   // 0 for an empty one
        Z = fmaf(f, dep_l[u * kGroup + h], Z);
        const float* src = dep_o + (u * kGroup + h) * kHeadDim + d;
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] = fmaf(f, src[i], acc[i]);
      }
    }
    const float f = M == -INFINITY ? 0.f : (P.v_scale && F::kScaled ? P.v_scale[kvh_done] : 1.f) / Z;
    const long long row = (long long)b_done * (P.Hkv * kGroup) + head;
    if (P.out_f32) {
      float* dst = P.out_f32 + row * kHeadDim + d;
#pragma unroll
      for (int i = 0; i < VEC; ++i) dst[i] = acc[i] * f;
    } else {
      __nv_bfloat16* dst = P.out + row * kHeadDim + d;
      if constexpr (VEC == 1) {
        dst[0] = __float2bfloat16_rn(acc[0] * f);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; i += 2)
          reinterpret_cast<uint32_t*>(dst)[i / 2] = f32x2_to_bf16x2(acc[i] * f, acc[i + 1] * f);
      }
    }
    if (d == 0 && P.lse_out) P.lse_out[row] = Z != 0.f ? (M + log2f(Z)) * 0.6931471805599453f : -INFINITY;
    group_sync<GW>(group);   // the deposits have been read
  }
}

template <int GW>
static cudaError_t launch_group_variant(const DecodeParams& P, int ctas, cudaStream_t s, int& smem_limit) {
  auto kern = decode_attn_group_kernel<GW, Fp4Tile>;
  constexpr size_t need = Fp4Tile::kAlign +
                          (size_t)kGrpWarps * kGrpStages * 2 * (kGrpTile / kBlock) * Fp4Tile::kBlockBytes +
                          (size_t)kGrpWarps * kGroup * (kHeadDim + 2) * sizeof(float) + kGrpWarps * kGrpStages * 8;
  if (smem_limit == 0) {  // first launch of this variant on this device: raise its dynamic shared-memory limit
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)need);
    if (e != cudaSuccess) return e;
    smem_limit = (int)need;
  }
  return launch_dependent(kern, dim3(ctas), dim3(kGrpWarps * 32), need, s, P);
}

cudaError_t launch_decode_attn_group(const DecodeParams& P, int warps, int ctas, cudaStream_t s, int* smem_limit) {
  switch (warps) {
    case 1: return launch_group_variant<1>(P, ctas, s, smem_limit[0]);
    case 2: return launch_group_variant<2>(P, ctas, s, smem_limit[1]);
    case 4: return launch_group_variant<4>(P, ctas, s, smem_limit[2]);
    case 8: return launch_group_variant<8>(P, ctas, s, smem_limit[3]);
    default: return launch_group_variant<16>(P, ctas, s, smem_limit[4]);
  }
}

}  // namespace puzzle
