// Decode attention over the 4-bit cache: the group kernel, for one query token per sequence and for pairs of them.
//
// A group of GW warps takes a run of tiles of one (sequence, KV head) pair, warp i of the group the tiles i, i + GW, ... of
// the run, and the warps' states meet in shared memory at its end.  Compared with a warp as the worker (decode_attn.cu)
// there are GW times fewer partials; compared with tiles handed out inside a CTA (decode_attn_cta.cu) nothing is
// claimed or recorded per tile.  Both weigh more here than on the E4M3 cache: a 4-bit tile has half the bytes of an E4M3
// tile and as many instructions, so what a tile costs besides its arithmetic decides (CTA-balanced kernel 123 us at 16 x
// 64K, 143 at 37 x 32K; this one 117 and 130).  Comparisons in this file are of launches without pause on one GPU; these run at
// the power cap, and what the codes are decides with: 16 x 64K takes 112 us over normally distributed values, 128 over
// uniformly random codes.
//  * Whole pairs: a launch that fills the SMs evenly needs no cutting.  No schedule is built, nothing but inputs and
//    outputs touches global memory, and the end of a pair is one barrier of its group.  4 x 1024 tokens 6.1 us (evenly cut
//    over all warps 13.9), 16 x 4096 11.7 (20.2), 16 x 16384 34.5 (44).
//  * CUT: the tile space of all pairs is cut evenly over the groups; a run that is not a whole pair leaves one float32
//    partial, and a small second kernel merges them.
// The tile loop of one token takes 122 registers without spilling, so sixteen warps fit; a pair of tokens 162 to 166, twelve.
// At 16 x 64K the kernel reads 5.2 to 5.4 TB/s.  Bare copies of the same blocks in the same order run at 5.9 (6.5 when the blocks of
// two heads are fetched together: a block of one head is 576 bytes); the rest is the arithmetic, which alone would take
// about 105 us, and 10 us of set-up, first tile and merge.
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
    int prow;                // first partial row of this run, or -1: the run is the whole pair
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
    int prow;
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

// cum[1 .. n] -> their prefix sums, by the CTA's first warp; ends with a CTA barrier.
__device__ __forceinline__ void prefix_sum(int* cum, int n) {
  if (threadIdx.x < 32) {
    int carry = 0;
    for (int base = 0; base < n; base += 32) {
      const int i = base + threadIdx.x;
      int v = i < n ? cum[i + 1] : 0;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, v, d);
        if ((int)threadIdx.x >= d) v += u;
      }
      if (i < n) cum[i + 1] = v + carry;
      carry += __shfl_sync(0xffffffffu, v, 31);
    }
  }
  __syncthreads();
}

template <int GW>
__device__ __forceinline__ void group_sync(int group) {
  if constexpr (GW == 1) __syncwarp();
  else asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(GW * 32) : "memory");
}

}  // namespace

// Q: OneToken or TokenPair.  CUT: the tile space of all pairs is cut evenly over the groups, and a run that is not a whole
// pair leaves a partial; else groups take whole pairs.
template <int GW, typename Q, bool CUT>
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
  const uint32_t bars = smem_u32(sp) + warp * (NS * 8);             sp += NW * NS * 8;
  int* cum = reinterpret_cast<int*>(sp);   // CUT: tiles of all KV heads of the rows before row i
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
  const int rows = Q::rows(P), pairs = rows * P.Hkv, step = gridDim.x * NG;
  // WHOLE: next pair; neighbouring pairs on different SMs.  CUT: [pos, end) of the tile space, `share` tiles per group
  int pos = group * gridDim.x + blockIdx.x, end = pairs, share = 0;
  if constexpr (CUT) {
    if (threadIdx.x == 0) cum[0] = 0;
    for (int i = threadIdx.x; i < rows; i += blockDim.x) {
      typename Q::Item it;
      Q::item(P, i, it);
      if (it.too_long && P.dev_status && blockIdx.x == 0) atomicOr(P.dev_status, (int)PUZZLE_DEV_SEQ_TOO_LONG);
      cum[i + 1] = (it.t_end - it.t0) * P.Hkv;
    }
    __syncthreads();
    prefix_sum(cum, rows);
    const int T = cum[rows];
    share = (T + step - 1) / step;
    pos = min((int)(blockIdx.x * NG + group) * share, T);
    end = min(pos + share, T);
    // pairs without any visible key have no tile and hence no run: the merge writes their outputs
    for (int p = blockIdx.x * blockDim.x + threadIdx.x; p < pairs; p += gridDim.x * blockDim.x)
      if (cum[p / P.Hkv + 1] == cum[p / P.Hkv]) P.pair_parts[p] = make_int2(0, 0);
  }

  // ---- the pair whose tiles are issued and computed, and this warp's copies: two tiles ahead, table entries three
  typename Q::Item it{};
  int t_issue, phys;     // next tile to issue, and its blocks (lane i < NB: block i)
  int j_lo, j_n;         // one token: blocks [j_lo, j_lo + j_n) of the sequence are fetched
  const int32_t* table;  // one token: the sequence's row of the block table, or null
  int stage = 0;
  uint32_t phase = 0;
  bool failed = false;   // a copy did not land in time: this warp stops computing but keeps in step with its group
  auto lookup = [&]() {
    phys = INT_MIN;
    const int j = t_issue * NB + lane;
    // The same range, with what a run has in common worked out at its start: 2.4 % less time at 16 x 64K, 3.6 % at 37 x 32K
    // (123.5 to 120.5 us, 137 to 132).  For a pair of tokens the registers it takes cost more (twelve-warp groups: 155 to 169 us at 16 x 64K).
    if constexpr (Q::kTokens == 1) {
      if (lane < NB && (unsigned)(j - j_lo) < (unsigned)j_n) phys = table ? table[j] : it.b * P.max_blocks_per_seq + j;
    } else {
      if (t_issue < it.t_end && lane < NB && j * kBlock < it.L && j * kBlock + kBlock > it.loA)
        phys = P.block_table ? P.block_table[(size_t)it.b * P.max_blocks_per_seq + j] : it.b * P.max_blocks_per_seq + j;
    }
  };
  auto issue = [&](int st) {
    if (t_issue >= it.t_end) return;
    int row = P.oob_row;
    if (lane < NB) {
      if (Q::kTokens == 1 ? (unsigned)phys < (unsigned)P.num_blocks : phys >= 0 && phys < P.num_blocks)   // < 2^31: check_view
        row = phys * P.Hkv + it.kvh;   // the maps have one row per block and head
      else if (phys != INT_MIN && P.dev_status) atomicOr(P.dev_status, (int)PUZZLE_DEV_BAD_BLOCK);
    }
    F::template load_tile<NB>(P, pipe + st * STAGE_BYTES, row, bars + 8 * st);
    t_issue += GW;
    lookup();
  };
  // The next run and its first copies; all earlier tiles of this warp have been consumed.
  auto start = [&]() -> bool {
    if (pos >= end) return false;
    if constexpr (CUT) {
      int a = 0, z = rows;   // the row the position falls into
      while (z - a > 1) {
        const int mid = (a + z) >> 1;
        if (cum[mid] <= pos) a = mid; else z = mid;
      }
      Q::item(P, a, it);
      const int nt = it.t_end - it.t0, first = cum[a];
      it.kvh = (pos - first) / nt;
      const int g0 = first + it.kvh * nt, stop = min(g0 + nt, end), p = a * P.Hkv + it.kvh;
      const int w0 = g0 / share, parts = (g0 + nt - 1) / share - w0 + 1;
      it.prow = parts == 1 ? -1 : ((int)(blockIdx.x * NG + group) + p) * (Q::kTokens * kGroup);
      if (pos == g0 && wi == 0 && lane == 0)   // the group with a pair's first tile tells the merge where its partials are
        P.pair_parts[p] = make_int2((w0 + p) * (Q::kTokens * kGroup), parts == 1 ? -1 : parts);
      it.t0 += pos - g0;
      it.t_end = it.t0 + (stop - pos);
      pos = stop;
    } else {
      const int row = pos / P.Hkv;
      Q::item(P, row, it);
      it.kvh = pos - row * P.Hkv;
      it.prow = -1;
      if (it.too_long && P.dev_status && it.kvh == 0 && wi == 0 && lane == 0)
        atomicOr(P.dev_status, (int)PUZZLE_DEV_SEQ_TOO_LONG);
      pos += step;
    }
    t_issue = failed ? it.t_end : it.t0 + wi;
    if constexpr (Q::kTokens == 1) {
      table = P.block_table ? P.block_table + (size_t)it.b * P.max_blocks_per_seq : nullptr;
      j_lo = it.lo / kBlock;
      j_n = max(0, min((it.L + kBlock - 1) / kBlock, it.t_end * NB) - j_lo);
    }
    lookup();
#pragma unroll
    for (int i = 0; i < NS; ++i) issue((stage + i) % NS);
    return true;
  };

  bool more = start();
#pragma unroll 1
  while (more) {
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
    more = start();   // the next run's first tiles are on their way while this one is combined

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
      const bool part = CUT && done.prow >= 0;
      // the group's threads take two adjacent output values each, in as many turns as it needs
#pragma unroll 1
      for (int e = 2 * (wi * 32 + lane); e < kGroup * kHeadDim && first >= 0; e += 2 * GW * 32) {
        const int h = e / kHeadDim, d = e % kHeadDim;
        const int head = done.kvh * kGroup + h;
        const float sink = P.sinks && !part ? P.sinks[head] * 1.4426950408889634f : -INFINITY;
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
        const long long row = part ? (long long)done.prow + tok * kGroup + h : first + head;
        float* f32 = part ? P.part_o : P.out_f32;
        float* lse = part ? P.part_lse : P.lse_out;
        if (f32) *reinterpret_cast<float2*>(f32 + row * kHeadDim + d) = make_float2(a0 * f, a1 * f);
        else *reinterpret_cast<uint32_t*>(P.out + row * kHeadDim + d) = f32x2_to_bf16x2(a0 * f, a1 * f);
        if (d == 0 && lse) lse[row] = Z != 0.f ? (M + log2f(Z)) * 0.6931471805599453f : -INFINITY;
      }
      group_sync<GW>(group);   // the deposits have been read
    }
  }
}

// The partials of the pairs that were cut, one warp per (pair, token): the quad of lanes g owns query head g of the group,
// lane c of the quad channels 16c .. 16c + 15.  The formula is merge_rows' (decode_sched.cuh); four parts per round, all
// their loads before the first use.  A kernel of its own, launched as a dependent: merging inside the attention kernel
// takes fences, arrival counters and registers of its tile loop (124 to 136 us against 117 at 16 x 64K).
template <typename Q>
__global__ void __launch_bounds__(128) decode_attn_parts_kernel(const __grid_constant__ DecodeParams P) {
  const int item = (blockIdx.x * blockDim.x + threadIdx.x) >> 5, lane = threadIdx.x & 31;
  const int p = item / Q::kTokens, tok = item - p * Q::kTokens;
  const int g = lane >> 2, c = lane & 3;
  release_dependents();
  grid_dependency_wait();
  if (p >= Q::rows(P) * P.Hkv) return;
  const int2 parts = P.pair_parts[p];
  if (parts.y < 0) return;   // one group had the whole pair and has written it
  typename Q::Item it{};
  Q::item(P, p / P.Hkv, it);
  const long long first = Q::row_out(P, it, tok);
  if (first < 0) return;
  const int head = (p % P.Hkv) * kGroup + g;
  const float sink = P.sinks ? P.sinks[head] : -INFINITY;
  const long long base = (long long)parts.x + tok * kGroup + g;
  constexpr int kStride = Q::kTokens * kGroup;
  float M = -INFINITY;
  for (int k = c; k < parts.y; k += 4) M = fmaxf(M, P.part_lse[base + (long long)k * kStride]);
  M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, 1));
  M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, 2));
  M = fmaxf(M, sink);
  float acc[16], Z = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
  if (M != -INFINITY) {
    if (sink != -INFINITY) Z = __expf(sink - M);   // the sink is one more softmax column, counted once
    for (int k0 = 0; k0 < parts.y; k0 += 4) {
      float l[4];
      float4 v[4][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool on = k0 + j < parts.y;
        const long long row = base + (long long)(on ? k0 + j : k0) * kStride;
        l[j] = on ? P.part_lse[row] : -INFINITY;
        const float4* o = reinterpret_cast<const float4*>(P.part_o + row * kHeadDim + 16 * c);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[j][i] = o[i];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (l[j] == -INFINITY) continue;
        const float wgt = __expf(l[j] - M);
        Z += wgt;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[4 * i + 0] += wgt * v[j][i].x; acc[4 * i + 1] += wgt * v[j][i].y;
          acc[4 * i + 2] += wgt * v[j][i].z; acc[4 * i + 3] += wgt * v[j][i].w;
        }
      }
    }
  }
  const float f = M == -INFINITY ? 0.f : 1.f / Z;
  const long long row = first + head;
  if (P.out_f32) {
    float4* dst = reinterpret_cast<float4*>(P.out_f32 + row * kHeadDim + 16 * c);
#pragma unroll
    for (int i = 0; i < 4; ++i) dst[i] = make_float4(acc[4 * i] * f, acc[4 * i + 1] * f, acc[4 * i + 2] * f, acc[4 * i + 3] * f);
  } else {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = f32x2_to_bf16x2(acc[2 * i] * f, acc[2 * i + 1] * f);
    uint4* dst = reinterpret_cast<uint4*>(P.out + row * kHeadDim + 16 * c);
    dst[0] = make_uint4(w[0], w[1], w[2], w[3]);
    dst[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
  if (P.lse_out && c == 0) P.lse_out[row] = Z != 0.f ? M + __logf(Z) : -INFINITY;
}

template <int GW, typename Q, bool CUT>
static cudaError_t launch_group_variant(const DecodeParams& P, int ctas, cudaStream_t s, int& smem_limit) {
  auto kern = decode_attn_group_kernel<GW, Q, CUT>;
  constexpr size_t fixed = Fp4Tile::kAlign +
                           (size_t)Q::kWarps * kGrpStages * 2 * (kGrpTile / kBlock) * Fp4Tile::kBlockBytes +
                           (size_t)Q::kWarps * kGroup * (kHeadDim + 2) * sizeof(float) + Q::kWarps * kGrpStages * 8;
  const int rows = P.batch * (Q::kTokens == 2 ? (P.n_q + 1) / 2 : 1);
  const size_t need = fixed + (CUT ? (size_t)(rows + 1) * sizeof(int) : 0);
  if (smem_limit == 0) {  // first launch of this variant on this device: raise its dynamic shared-memory limit
    int dev = 0, optin = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, optin);
    if (e != cudaSuccess) return e;
    smem_limit = optin;
  }
  if (need > (size_t)smem_limit) return cudaErrorInvalidValue;   // too many rows for the schedule array
  cudaError_t e = launch_dependent(kern, dim3(ctas), dim3(Q::kWarps * 32), need, s, P);
  if (CUT && e == cudaSuccess) {
    count_launch();
    const long long warps = (long long)rows * P.Hkv * Q::kTokens;
    e = launch_dependent(decode_attn_parts_kernel<Q>, dim3((unsigned)((warps + 3) / 4)), dim3(128), 0, s, P);
  }
  return e;
}

template <bool CUT>
static cudaError_t launch_one(const DecodeParams& P, int warps, int ctas, cudaStream_t s, int* smem_limit) {
  if constexpr (!CUT) {   // cut launches have groups of four warps or more
    if (warps == 1) return launch_group_variant<1, OneToken, CUT>(P, ctas, s, smem_limit[0]);
    if (warps == 2) return launch_group_variant<2, OneToken, CUT>(P, ctas, s, smem_limit[1]);
  }
  switch (warps) {
    case 4: return launch_group_variant<4, OneToken, CUT>(P, ctas, s, smem_limit[2]);
    case 8: return launch_group_variant<8, OneToken, CUT>(P, ctas, s, smem_limit[3]);
    default: return launch_group_variant<16, OneToken, CUT>(P, ctas, s, smem_limit[4]);
  }
}
cudaError_t launch_decode_attn_group(const DecodeParams& P, int warps, bool cut, int ctas, cudaStream_t s, int* smem_limit) {
  return cut ? launch_one<true>(P, warps, ctas, s, smem_limit + 5) : launch_one<false>(P, warps, ctas, s, smem_limit);
}

template <bool CUT>
static cudaError_t launch_pair(const DecodeParams& P, int warps, int ctas, cudaStream_t s, int* smem_limit) {
  if constexpr (!CUT) {
    if (warps == 1) return launch_group_variant<1, TokenPair, CUT>(P, ctas, s, smem_limit[0]);
    if (warps == 2) return launch_group_variant<2, TokenPair, CUT>(P, ctas, s, smem_limit[1]);
  }
  switch (warps) {
    case 4: return launch_group_variant<4, TokenPair, CUT>(P, ctas, s, smem_limit[2]);
    case 6: return launch_group_variant<6, TokenPair, CUT>(P, ctas, s, smem_limit[3]);
    default: return launch_group_variant<12, TokenPair, CUT>(P, ctas, s, smem_limit[4]);
  }
}
cudaError_t launch_decode_attn_tokens_group(const DecodeParams& P, int warps, bool cut, int ctas, cudaStream_t s,
                                            int* smem_limit) {
  return cut ? launch_pair<true>(P, warps, ctas, s, smem_limit + 5) : launch_pair<false>(P, warps, ctas, s, smem_limit);
}

}  // namespace puzzle
