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
#include "decode_tokens.cuh"

namespace puzzle {
namespace {

constexpr int kGrpStages = 2, kGrpTile = kTokTile;

// What a group works on: a (sequence, KV head) pair with one query token ...
struct OneToken {
  static constexpr int kTokens = 1, kWarps = 16;
  using Tile = Fp4Tile;
  using State = Fp4State;
  struct Item {
    int b, kvh, t0, t_end;   // tiles [t0, t_end)
    int L, lo;               // keys [lo, L) are visible
    bool too_long;
  };
  static __device__ __forceinline__ int rows(const DecodeParams& P) { return P.batch; }
  static __device__ __forceinline__ void item(const DecodeParams& P, int row, Item& it) {
    const SeqRange r = seq_range(P.seq_lens[row], P.window, P.max_blocks_per_seq * kBlock, kGrpTile, it.too_long);
    it.b = row; it.L = r.L; it.lo = r.lo; it.t0 = r.tlo; it.t_end = r.tlo + r.ntile;
  }
  static __device__ __forceinline__ void load_query(State& st, const DecodeParams& P, const Item& it, float ks, int lane) {
    st.load_query(P.q + ((size_t)it.b * (P.Hkv * kGroup) + it.kvh * kGroup + (lane >> 2)) * kHeadDim, ks, P.sm_scale_log2e, lane);
  }
  static __device__ __forceinline__ void tile(State& st, const Fp4Lanes& at, uint32_t kbase, uint32_t vbase, int tok0,
                                              const Item& it, int lane) {
    if (tok0 < it.lo || tok0 + kGrpTile > it.L) Fp4Tile::tile<kGrpTile, true>(st, at, kbase, vbase, tok0, it.lo, it.L, lane);
    else Fp4Tile::tile<kGrpTile, false>(st, at, kbase, vbase, tok0, it.lo, it.L, lane);
  }
  static __device__ __forceinline__ void finish(const State& st, int, float& m, float& l, float (&o)[8][2], int lane) {
    Fp4Tile::finish(st, m, l, o, lane);
  }
  // Output row of head 0 of the sequence (token tok), or -1.
  static __device__ __forceinline__ long long row_out(const DecodeParams& P, const Item& it, int) {
    return (long long)it.b * (P.Hkv * kGroup);
  }
};

// ... or with two (a row of the multi-token schedule).  Twelve warps: two tokens' accumulators take 162 registers.
struct TokenPair {
  static constexpr int kTokens = 2, kWarps = 12;
  using Tile = Fp4Tile;
  using State = Fp4Pair::State;
  struct Item {
    int b, kvh, t0, t_end;
    int L, lo;               // keys [lo, L) are visible to the later token; table entries are needed from loA on
    int LA, loA, tok, odd;   // the earlier token: keys [loA, LA), index tok; odd: there is no second token
    bool too_long;
  };
  static __device__ __forceinline__ int rows(const DecodeParams& P) { return P.batch * ((P.n_q + 1) >> 1); }
  static __device__ __forceinline__ void item(const DecodeParams& P, int row, Item& it) {
    const RowInfo i = row_info(P, row);
    it.b = i.b; it.L = i.L; it.lo = i.lo; it.LA = i.LA; it.loA = i.loA;
    it.tok = i.present ? i.t0 : -1;
    it.odd = i.t1 == i.t0;
    it.t0 = i.tlo; it.t_end = i.tlo + i.ntile;
    it.too_long = i.too_long;
  }
  static __device__ __forceinline__ void load_query(State& st, const DecodeParams& P, const Item& it, float ks, int lane) {
    const int Hq = P.Hkv * kGroup;
    const __nv_bfloat16* q = P.q + (((size_t)it.b * P.n_q + it.tok) * Hq + it.kvh * kGroup + (lane >> 2)) * kHeadDim;
    Fp4Pair::load_query(st, 0, q, ks, P.sm_scale_log2e, lane);
    Fp4Pair::load_query(st, 1, it.odd ? q : q + (size_t)Hq * kHeadDim, ks, P.sm_scale_log2e, lane);
  }
  static __device__ __forceinline__ void tile(State& st, const Fp4Lanes& at, uint32_t kbase, uint32_t vbase, int tok0,
                                              const Item& it, int lane) {
    if (tok0 < it.lo || tok0 + kGrpTile > it.LA)
      Fp4Pair::tile<true>(st, at, kbase, vbase, tok0, it.loA, it.LA, it.lo, it.L, lane);
    else Fp4Pair::tile<false>(st, at, kbase, vbase, tok0, it.loA, it.LA, it.lo, it.L, lane);
  }
  static __device__ __forceinline__ void finish(const State& st, int tok, float& m, float& l, float (&o)[8][2], int lane) {
    Fp4Tile::finish(st.t[tok], m, l, o, lane);
  }
  static __device__ __forceinline__ long long row_out(const DecodeParams& P, const Item& it, int tok) {
    if (it.tok < 0 || (tok == 1 && it.odd)) return -1;   // rows behind the last token stay as they are
    return ((long long)it.b * P.n_q + it.tok + tok) * (P.Hkv * kGroup);
  }
};

template <int GW>
__device__ __forceinline__ void group_sync(int group) {
  if constexpr (GW == 1) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(GW * 32) : "memory");
}

}  // namespace

// Q: OneToken or TokenPair.
template <int GW, typename Q>
__global__ void __launch_bounds__(Q::kWarps * 32, 1) decode_attn_group_kernel(const __grid_constant__ DecodeParams P) {
  using F = typename Q::Tile;
  constexpr int NW = Q::kWarps, NS = kGrpStages, TT = kGrpTile, NB = TT / kBlock, NG = NW / GW;
  constexpr int STAGE_BYTES = 2 * NB * F::kBlockBytes;
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
  const int pairs = Q::rows(P) * P.Hkv, step = gridDim.x * NG;

  // ---- the pair whose tiles are issued and computed, and this warp's copies: two tiles ahead, table entries three
  typename Q::Item it;
  int t_issue, phys;     // next tile to issue, and its blocks (lane i < NB: block i)
  int stage = 0;
  uint32_t phase = 0;
  bool failed = false;   // a copy did not land in time: this warp stops computing but keeps in step with its group
  auto lookup = [&]() {
    phys = INT_MIN;
    const int j = t_issue * NB + lane;
    int lo = it.lo;
    if constexpr (Q::kTokens == 2) lo = it.loA;
    if (t_issue < it.t_end && lane < NB && j * kBlock < it.L && j * kBlock + kBlock > lo)
      phys = P.block_table ? P.block_table[(size_t)it.b * P.max_blocks_per_seq + j] : it.b * P.max_blocks_per_seq + j;
  };
  auto issue = [&](int st) {
    if (t_issue >= it.t_end) return;
    int row = P.oob_row;
    if (lane < NB) {
      if (phys >= 0 && phys < P.num_blocks) row = (phys * P.Hkv + it.kvh) * P.rows_per_block;
      else if (phys != INT_MIN && P.dev_status) atomicOr(P.dev_status, (int)PUZZLE_DEV_BAD_BLOCK);
    }
    F::template load_tile<NB>(P, pipe + st * STAGE_BYTES, row, bars + 8 * st, lane, [] {});
    t_issue += GW;
    lookup();
  };
  auto start = [&](int p) {   // the pair and its first copies; all earlier tiles of this warp have been consumed
    const int row = p / P.Hkv;
    Q::item(P, row, it);
    it.kvh = p - row * P.Hkv;
    if (it.too_long && P.dev_status && it.kvh == 0 && wi == 0 && lane == 0)
      atomicOr(P.dev_status, (int)PUZZLE_DEV_SEQ_TOO_LONG);
    t_issue = failed ? it.t_end : it.t0 + wi;
    lookup();
#pragma unroll
    for (int i = 0; i < NS; ++i) issue((stage + i) % NS);
  };

  int p = group * gridDim.x + blockIdx.x;   // neighbouring pairs on different SMs
  if (p < pairs) start(p);
#pragma unroll 1
  while (p < pairs) {
    typename Q::State st;
    st.reset();
    if (it.t0 + wi < it.t_end) Q::load_query(st, P, it, P.k_scale && F::kScaled ? P.k_scale[it.kvh] : 1.f, lane);
#pragma unroll 1
    for (int t = it.t0 + wi; t < it.t_end && !failed; t += GW) {
      if (!mbar_wait_bounded(bars + 8 * stage, phase)) {
        if (P.dev_status && lane == 0) atomicOr(P.dev_status, (int)PUZZLE_DEV_WAIT_EXPIRED);
        failed = true;
        // the other copy in flight gets a bounded chance to land: nothing of this warp is under way when it goes on
        if (t + GW < t_issue) mbar_wait_bounded(bars + 8 * (stage ^ 1), phase ^ (uint32_t)stage);
        break;
      }
      const uint32_t kbase = pipe + stage * STAGE_BYTES, vbase = kbase + NB * F::kBlockBytes;
      Q::tile(st, at, kbase, vbase, t * TT, it, lane);
      __syncwarp();
      issue(stage);
      if (++stage == NS) { stage = 0; phase ^= 1u; }
    }
    const typename Q::Item done = it;
    p += step;
    if (p < pairs) start(p);   // the next pair's first tiles are on their way while this one is combined

    const int parts = min(done.t_end - done.t0, GW);
    const float vs = P.v_scale && F::kScaled ? P.v_scale[done.kvh] : 1.f;
#pragma unroll
    for (int tok = 0; tok < Q::kTokens; ++tok) {
      // ---- the warps' states meet; one without a tile leaves an empty one
      float m, l, o[8][2];
      Q::finish(st, tok, m, l, o, lane);
      F::store(dep_o + (wi * kGroup + g) * kHeadDim, o, 1.f, c);
      if (c == 0) {
        dep_m[wi * kGroup + g] = l == 0.f ? -INFINITY : m;
        dep_l[wi * kGroup + g] = l;
      }
      group_sync<GW>(group);
      const long long first = Q::row_out(P, done, tok);
      // the group's threads take two adjacent output values each, in as many turns as it needs
#pragma unroll 1
      for (int e = 2 * (wi * 32 + lane); e < kGroup * kHeadDim && first >= 0; e += 2 * GW * 32) {
        const int h = e / kHeadDim, d = e % kHeadDim;
        const int head = done.kvh * kGroup + h;
        const float sink = P.sinks ? P.sinks[head] * 1.4426950408889634f : -INFINITY;
        float M = sink, Z = 0.f, a0 = 0.f, a1 = 0.f;
        for (int u = 0; u < parts; ++u) M = fmaxf(M, dep_m[u * kGroup + h]);
        if (M != -INFINITY) {
          Z = sink == -INFINITY ? 0.f : ex2(sink - M);
          for (int u = 0; u < parts; ++u) {
            const float f = ex2(dep_m[u * kGroup + h] - M);   // 0 for an empty one
            Z = fmaf(f, dep_l[u * kGroup + h], Z);
            const float2 v = *reinterpret_cast<const float2*>(dep_o + (u * kGroup + h) * kHeadDim + d);
            a0 = fmaf(f, v.x, a0);
            a1 = fmaf(f, v.y, a1);
          }
        }
        const float f = M == -INFINITY ? 0.f : vs / Z;
        const long long at_out = (first + head) * kHeadDim + d;
        if (P.out_f32) *reinterpret_cast<float2*>(P.out_f32 + at_out) = make_float2(a0 * f, a1 * f);
        else *reinterpret_cast<uint32_t*>(P.out + at_out) = f32x2_to_bf16x2(a0 * f, a1 * f);
        if (d == 0 && P.lse_out) P.lse_out[first + head] = Z != 0.f ? (M + log2f(Z)) * 0.6931471805599453f : -INFINITY;
      }
      group_sync<GW>(group);   // the deposits have been read
    }
  }
}

template <int GW, typename Q>
static cudaError_t launch_group_variant(const DecodeParams& P, int ctas, cudaStream_t s, int& smem_limit) {
  auto kern = decode_attn_group_kernel<GW, Q>;
  constexpr size_t need = Fp4Tile::kAlign +
                          (size_t)Q::kWarps * kGrpStages * 2 * (kGrpTile / kBlock) * Fp4Tile::kBlockBytes +
                          (size_t)Q::kWarps * kGroup * (kHeadDim + 2) * sizeof(float) + Q::kWarps * kGrpStages * 8;
  if (smem_limit == 0) {  // first launch of this variant on this device: raise its dynamic shared-memory limit
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)need);
    if (e != cudaSuccess) return e;
    smem_limit = (int)need;
  }
  return launch_dependent(kern, dim3(ctas), dim3(Q::kWarps * 32), need, s, P);
}

cudaError_t launch_decode_attn_group(const DecodeParams& P, int warps, int ctas, cudaStream_t s, int* smem_limit) {
  switch (warps) {
    case 1: return launch_group_variant<1, OneToken>(P, ctas, s, smem_limit[0]);
    case 2: return launch_group_variant<2, OneToken>(P, ctas, s, smem_limit[1]);
    case 4: return launch_group_variant<4, OneToken>(P, ctas, s, smem_limit[2]);
    case 8: return launch_group_variant<8, OneToken>(P, ctas, s, smem_limit[3]);
    default: return launch_group_variant<16, OneToken>(P, ctas, s, smem_limit[4]);
  }
}

cudaError_t launch_decode_attn_tokens_group(const DecodeParams& P, int warps, int ctas, cudaStream_t s, int* smem_limit) {
  switch (warps) {
    case 1: return launch_group_variant<1, TokenPair>(P, ctas, s, smem_limit[0]);
    case 2: return launch_group_variant<2, TokenPair>(P, ctas, s, smem_limit[1]);
    case 4: return launch_group_variant<4, TokenPair>(P, ctas, s, smem_limit[2]);
    case 6: return launch_group_variant<6, TokenPair>(P, ctas, s, smem_limit[3]);
    default: return launch_group_variant<12, TokenPair>(P, ctas, s, smem_limit[4]);
  }
}

}  // namespace puzzle
