// Host side of the C ABI declared in include/puzzle_attn.h: argument checks, TMA descriptor
// encoding and kernel launches.  No allocation, no synchronisation, no state besides a launch counter.
#include <algorithm>
#include <atomic>
#include <cstring>

#include "common.cuh"
#include "decode_attn.cuh"

namespace puzzle {

static std::atomic<long long> g_launches{0};
void count_launch() { g_launches.fetch_add(1, std::memory_order_relaxed); }

namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_tiled() {
  static EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) != cudaSuccess ||
        qres != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}

// Whether the `bytes` bytes at p lie in one page-locked allocation.  Allocations of their own can follow each other without a
// gap, and a copy may not cross from one into the next.  Pageable memory: false.
bool one_pinned_range(const void* p, size_t bytes) {
  typedef CUresult (*Attributes)(unsigned int, CUpointer_attribute*, void**, CUdeviceptr);
  static Attributes get = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuPointerGetAttributes", &f, cudaEnableDefault, &qres) != cudaSuccess ||
        qres != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<Attributes>(f);
  }();
  if (!get) return false;
  CUdeviceptr start = 0;
  size_t size = 0;
  CUpointer_attribute what[2] = {CU_POINTER_ATTRIBUTE_RANGE_START_ADDR, CU_POINTER_ATTRIBUTE_RANGE_SIZE};
  void* into[2] = {&start, &size};
  const CUdeviceptr at = reinterpret_cast<CUdeviceptr>(p);
  return get(2, what, into, at) == CUDA_SUCCESS && size != 0 && start <= at && at + bytes <= start + size;
}

struct DeviceInfo {
  int sm_count = 0;
  // dynamic shared-memory limits already set per kernel and cache type; 0 = not raised yet
  int smem_warp[3] = {}, smem_cta[2] = {}, smem_small[3] = {};
  int smem_tc = 0, smem_tokens = 0, smem_group[10] = {}, smem_tokens_group[10] = {};
};
DeviceInfo& device_info() {
  static DeviceInfo info[64];
  int dev = 0;
  cudaGetDevice(&dev);
  DeviceInfo& d = info[dev & 63];
  if (d.sm_count == 0) cudaDeviceGetAttribute(&d.sm_count, cudaDevAttrMultiProcessorCount, dev);
  return d;
}

puzzle_status check_desc(const puzzle_layer_desc* d) {
  if (!d) return PUZZLE_ERR_NULL;
  if (d->num_q_heads <= 0 || d->num_kv_heads <= 0 || d->head_dim <= 0 || d->block_size <= 0 || d->window < 0)
    return PUZZLE_ERR_SHAPE;
  if (d->num_q_heads % d->num_kv_heads != 0) return PUZZLE_ERR_SHAPE;
  if (d->kv_dtype != PUZZLE_KV_FP8_E4M3 && d->kv_dtype != PUZZLE_KV_BF16 && d->kv_dtype != PUZZLE_KV_FP4_E2M1)
    return PUZZLE_ERR_SHAPE;
  if (d->head_dim != kHeadDim || d->block_size != kBlock || d->num_q_heads != kGroup * d->num_kv_heads)
    return PUZZLE_ERR_UNSUPPORTED;
  return PUZZLE_OK;
}

puzzle_status check_view(const puzzle_layer_desc* d, const puzzle_kv_view* kv, int batch) {
  if (!kv || !kv->k_cache || !kv->v_cache || !kv->seq_lens) return PUZZLE_ERR_NULL;
  if (batch <= 0 || kv->num_blocks <= 0 || kv->max_blocks_per_seq <= 0) return PUZZLE_ERR_SHAPE;
  if (batch > kMaxBatch) return PUZZLE_ERR_UNSUPPORTED;
  if (kv->max_blocks_per_seq > (1 << 26)) return PUZZLE_ERR_UNSUPPORTED;   // tokens are counted in 32 bits, rounded up to tiles
  if ((reinterpret_cast<uintptr_t>(kv->k_cache) & 15) || (reinterpret_cast<uintptr_t>(kv->v_cache) & 15))
    return PUZZLE_ERR_SHAPE;
  // rows of the 2-D view of the cache must fit a signed 32-bit TMA coordinate
  if (kv->num_blocks * d->num_kv_heads * (long long)kBlock >= (1ll << 31) - 64) return PUZZLE_ERR_UNSUPPORTED;
  if (!kv->block_table && (long long)batch * kv->max_blocks_per_seq > kv->num_blocks) return PUZZLE_ERR_SHAPE;
  return PUZZLE_OK;
}

// 2-D view of a cache as rows of 128 bytes: two FP8 tokens or one bf16 token per row, so that every TMA
// request is a full 128-byte line.  Box = one 16-token block of one KV head (8 or 16 rows), 128-byte swizzle.
// row_bytes = 64 (FP8 only): one token per row, 16 rows per block, 64-byte swizzle (the tensor-memory kernel's view).
bool make_cache_map(CUtensorMap* m, void* base, long long rows, int elem_bytes, int row_bytes = 128) {
  EncodeTiledFn enc = encode_tiled();
  if (!enc) return false;
  if (row_bytes == 64) {
    const cuuint64_t dims[2] = {64, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {64};
    const cuuint32_t box[2] = {64, (cuuint32_t)kBlock};
    const cuuint32_t estr[2] = {1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
  }
  const cuuint64_t inner = 128 / elem_bytes;  // elements per row
  const cuuint64_t dims[2] = {inner, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {128};
  const cuuint32_t box[2] = {(cuuint32_t)inner, (cuuint32_t)(kBlock * kHeadDim * elem_bytes / 128)};
  const cuuint32_t estr[2] = {1, 1};
  CUresult r = enc(m, elem_bytes == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base,
                   dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                   CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS;
}

// 2-D view of a 4-bit cache: one row per (block, KV head), fetched four rows at a time (box of one row, as a gather
// wants it), unswizzled.
bool make_fp4_map(CUtensorMap* m, void* base, long long rows) {
  EncodeTiledFn enc = encode_tiled();
  if (!enc) return false;
  const cuuint64_t dims[2] = {PUZZLE_FP4_BLOCK_BYTES / 4, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {PUZZLE_FP4_BLOCK_BYTES};
  const cuuint32_t box[2] = {PUZZLE_FP4_BLOCK_BYTES / 4, 1};
  const cuuint32_t estr[2] = {1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_INT32, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a kernel reaches the cache: tensor maps of rows of row_bytes bytes (4-bit cache: of whole blocks).
bool set_cache(DecodeParams* P, const puzzle_layer_desc* d, const puzzle_kv_view* kv, int row_bytes) {
  if (d->kv_dtype == PUZZLE_KV_FP4_E2M1) {
    const long long rows = kv->num_blocks * d->num_kv_heads;
    P->rows_per_block = 1;
    P->oob_row = (int)rows;
    return make_fp4_map(&P->tmK, kv->k_cache, rows) && make_fp4_map(&P->tmV, kv->v_cache, rows);
  }
  const int eb = d->kv_dtype == PUZZLE_KV_FP8_E4M3 ? 1 : 2;
  P->rows_per_block = kBlock * kHeadDim * eb / row_bytes;
  const long long rows = kv->num_blocks * d->num_kv_heads * (long long)P->rows_per_block;
  P->oob_row = (int)rows;
  return make_cache_map(&P->tmK, kv->k_cache, rows, eb, row_bytes) && make_cache_map(&P->tmV, kv->v_cache, rows, eb, row_bytes);
}

constexpr int kMaxAppendHeads = 4096;   // the head groups of a chunk are a grid dimension
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// The parameters of an append that the descriptors hold; the rest is set by the entry points.
AppendParams append_params(const puzzle_layer_desc* d, const puzzle_kv_view* kv, int batch, int n_new,
                           const int32_t* new_lens, int32_t* dev_status) {
  AppendParams A;
  std::memset(&A, 0, sizeof A);
  A.k_cache = kv->k_cache;
  A.v_cache = kv->v_cache;
  A.block_table = kv->block_table;
  A.seq_lens = kv->seq_lens;
  A.new_lens = new_lens;
  A.k_scale = kv->k_scale;
  A.v_scale = kv->v_scale;
  A.dev_status = dev_status;
  A.num_blocks = kv->num_blocks;
  A.batch = batch;
  A.n_new = n_new;
  A.Hq = d->num_q_heads;
  A.Hkv = d->num_kv_heads;
  A.max_blocks_per_seq = kv->max_blocks_per_seq;
  return A;
}

// The plain append of contiguous k_new, v_new [batch][n_new][Hkv][D] to a 4-bit cache.
cudaError_t append_fp4(const puzzle_layer_desc* d, const puzzle_kv_view* kv, const void* k_new, const void* v_new,
                       const int32_t* new_lens, int batch, int n_new, int32_t* dev_status, cudaStream_t s) {
  AppendParams A = append_params(d, kv, batch, n_new, new_lens, dev_status);
  A.k = static_cast<const __nv_bfloat16*>(k_new);
  A.v = static_cast<const __nv_bfloat16*>(v_new);
  A.k_token_stride = A.v_token_stride = (long long)d->num_kv_heads * d->head_dim;
  A.k_seq_stride = A.v_seq_stride = A.k_token_stride * n_new;
  return launch_append(A, d->kv_dtype, false, false, s);
}

int grid_ctas() { return std::max(device_info().sm_count, 1); }

int decode_warps(int kv_dtype) {
  return kv_dtype == PUZZLE_KV_FP8_E4M3 ? kDecodeWarpsFp8 : (kv_dtype == PUZZLE_KV_BF16 ? kDecodeWarpsBf16 : kDecodeWarpsFp4);
}
int tile_tokens(int kv_dtype) {
  return kv_dtype == PUZZLE_KV_FP8_E4M3 ? kTileFp8 : (kv_dtype == PUZZLE_KV_BF16 ? kTileBf16 : kTileFp4);
}

// The workspace starts with the CTA-speed words of the CTA-balanced kernel, then one arrival counter per (sequence,
// KV head), then the partials.  Every completed call leaves the arrival counters at zero.  The counter block has room
// for kCounterFloor counters whatever the batch, so that up to that many (sequence, KV head) pairs the partials of
// one call never lie where another call's counters do: one prepared workspace then serves calls of different batch
// sizes one after the other.  Beyond the floor the layout follows the batch.
constexpr size_t kCounterFloor = 16384;
size_t cta_word_bytes() { return (cta_rate_words(grid_ctas()) * sizeof(int32_t) + 255) & ~(size_t)255; }
size_t counter_bytes(int batch, int Hkv) {
  const size_t n = std::max((size_t)batch * Hkv, kCounterFloor);
  return cta_word_bytes() + ((n * sizeof(int32_t) + 255) & ~(size_t)255);
}

// The balanced schedule runs on the CTA-balanced kernel when the batch fits its shared-memory schedule and the
// launch can be large: with at most a few tiles per warp (window layers, short contexts) a launch is a chain of
// latencies, which the warp-scheduled kernel's shorter set-up serves better.  The bound on the tiles comes from
// what the host knows: the window, or the length of a block-table row.
// Upper bound on the tiles of one (sequence, KV head) from what the host knows.
long long tiles_per_pair_bound(const puzzle_layer_desc* d, const puzzle_kv_view* kv) {
  const int tt = tile_tokens(d->kv_dtype);
  long long per_pair = ((long long)kv->max_blocks_per_seq * kBlock + tt - 1) / tt;
  if (d->window > 0) per_pair = std::min<long long>(per_pair, ((long long)d->window + tt - 1) / tt + 1);
  return per_pair;
}

bool use_cta_kernel(const puzzle_layer_desc* d, const puzzle_kv_view* kv, int batch, int num_splits) {
  if (num_splits == PUZZLE_SCHED_CTA) return true;
  if (num_splits != 0 || batch > kCtaMaxBatch) return false;
  // What the CTA-balanced kernel wins (no tail, CTAs cut by speed) grows with the length of the launch and of the
  // pairs; what it costs (a longer set-up, a claim and a hand-over per piece) weighs most on many short pairs.
  // Measured crossovers, in tiles per CTA: 64 with pairs of 256 tiles or more, about 200 at 128 tiles per pair,
  // about 600 below.
  const long long per_pair = tiles_per_pair_bound(d, kv);
  const long long min_per_cta = per_pair >= 256 ? kCtaMinTilesPerCta : (per_pair >= 128 ? 200 : 600);
  return per_pair * batch * d->num_kv_heads >= min_per_cta * grid_ctas();
}

// The kernel a call of puzzle_decode_attn runs on.
enum class Kernel { kCta, kWarp, kWarpWholePairs, kSmall, kGroup, kGroupCut };

// The 4-bit cache (times: uniform lengths, 148 SMs).  Groups that take whole pairs last as long as the SM with the most
// tiles, 4.5 us + 0.109 us a tile; groups that take even shares 15 us + 0.115 us per mean tile of an SM (the schedule, the
// partials and their merge are the difference).  Lengths may be ragged behind the bound the host has, so whole pairs have
// to promise a sixth, unless an SM gets many short ones whose sum evens out.  Whole / cut, us: 8 x 8192 tokens 17.9 / 19.8,
// 16 x 16384 34.5 / 39.7, 128 x 4096 62.7 / 67; but 1 x 16384 32 / 18, 8 x 32768 62 / 40, 24 x 30000 111 / 85.
bool whole_pairs_fp4(long long tiles, long long pairs) {
  const long long sms = grid_ctas(), per_sm = (pairs + sms - 1) / sms;
  return per_sm * tiles <= (pairs * tiles * 9) / (sms * 10) + 76 || (per_sm >= 5 && tiles <= 32);
}
Kernel pick_fp4_kernel(const puzzle_layer_desc* d, const puzzle_kv_view* kv, int batch) {
  const long long tiles = tiles_per_pair_bound(d, kv), pairs = (long long)batch * d->num_kv_heads;
  if (tiles <= kWholePairTiles && pairs <= decode_attn_small_max_pairs(grid_ctas())) return Kernel::kSmall;
  return whole_pairs_fp4(tiles, pairs) ? Kernel::kGroup : Kernel::kGroupCut;
}
// Warps per group.  Whole pairs: as many as leave every SM's sixteen warps a pair at once, fewer still when an SM has pairs
// to go round, where a smaller group waits less at their ends (512 x 1024 tokens: 4 warps 72.8 us, 2 65.2, 1 59.6; but a
// long pair is too coarse a share for one: 256 x 4096 114, 110, 116).  Cut: large groups leave few partials (1 x 65536: 16
// warps 22 us, 4 38), small ones few warps waiting at the ends of many runs (256 x 4096: 159, 122).
int group_warps(long long tiles, long long pairs, bool cut) {
  const long long n = (pairs + grid_ctas() - 1) / grid_ctas();
  if (cut) return n <= 1 ? 16 : n <= 4 ? 8 : 4;
  return n <= 1 ? 16 : n <= 2 ? 8 : n <= 4 ? 4 : (n <= 8 || tiles > 16) ? 2 : 1;
}
// The same for rows of two query tokens: 5 us + 0.155 us a tile against 20 us + 0.15 us, twelve warps.  (16 x 16384 tokens
// 47 us whole, 54 cut; 16 x 65536 161 / 152; 1 x 65536 156 / 34.)
bool whole_pairs_tokens(long long tiles, long long pairs) {
  const long long sms = grid_ctas(), per_sm = (pairs + sms - 1) / sms;
  return per_sm * tiles <= (pairs * tiles * 82) / (sms * 100) + 77 || (per_sm >= 5 && tiles <= 32);
}
int tokens_group_warps(long long tiles, long long pairs, bool cut) {
  const long long n = (pairs + grid_ctas() - 1) / grid_ctas();
  if (cut) return n <= 1 ? 12 : n <= 4 ? 6 : 4;
  return n <= 1 ? 12 : n <= 2 ? 6 : n <= 3 ? 4 : (n <= 6 || tiles > 16) ? 2 : 1;
}

Kernel pick_kernel(const puzzle_layer_desc* d, const puzzle_kv_view* kv, int batch, int num_splits) {
  if (d->kv_dtype == PUZZLE_KV_FP4_E2M1) {
    if (num_splits == PUZZLE_SCHED_CTA) return Kernel::kGroupCut;
    if (num_splits == 0) return pick_fp4_kernel(d, kv, batch);
  }
  if (use_cta_kernel(d, kv, batch, num_splits)) return Kernel::kCta;
  // Narrow windows and short contexts: with at most kWholePairTiles tiles per (sequence, KV head) a pair is not cut
  // at all.  A group of four warps (few pairs) or one warp (many pairs, or the warp-scheduled kernel pinned) takes
  // it whole and stores the output itself, which drops the partial, the arrival and the merge (three dependent
  // trips through L2) from a launch that is a chain of latencies anyway.
  const bool whole_pairs = num_splits <= 0 && tiles_per_pair_bound(d, kv) <= kWholePairTiles;
  if (!whole_pairs) return Kernel::kWarp;
  if (num_splits == 0 && (long long)batch * d->num_kv_heads <= decode_attn_small_max_pairs(grid_ctas()))
    return Kernel::kSmall;
  return Kernel::kWarpWholePairs;
}

size_t workspace_floats(int batch, int Hkv, int num_splits, int kv_dtype) {
  size_t rows;
  if (num_splits == 0) {
    // one row block per (worker, pair) meeting of the warp-scheduled kernels (the CTA-balanced kernel needs one
    // per (CTA, pair) meeting only, the tensor-memory kernel one per (worker, pair) with fewer workers)
    rows = ((size_t)grid_ctas() * decode_warps(kv_dtype) + (size_t)batch * Hkv) * kGroup;
  } else {
    rows = (size_t)batch * Hkv * kGroup * num_splits;
  }
  return rows * (kHeadDim + 1);
}
// Behind the partials of a 4-bit call: what the group kernel notes of every pair for its merge.
size_t pair_parts_bytes(size_t pairs, int kv_dtype) { return kv_dtype == PUZZLE_KV_FP4_E2M1 ? pairs * sizeof(int2) : 0; }

}  // namespace

// Everything about a decode-attention call that the host can check, short of the workspace.
puzzle_status check_decode_attn_args(const puzzle_layer_desc* desc, const puzzle_kv_view* kv, const void* q,
                                     const void* out, int batch, int num_splits, bool tcgen05) {
  puzzle_status st = check_desc(desc);
  if (st != PUZZLE_OK) return st;
  st = check_view(desc, kv, batch);
  if (st != PUZZLE_OK) return st;
  if (!q || !out) return PUZZLE_ERR_NULL;
  if (num_splits < PUZZLE_SCHED_WARP || num_splits > 65536) return PUZZLE_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(q) & 7) || (reinterpret_cast<uintptr_t>(out) & 15)) return PUZZLE_ERR_SHAPE;
  const bool fp4 = desc->kv_dtype == PUZZLE_KV_FP4_E2M1;   // its CTA-wide schedule has room for every batch
  if (num_splits == PUZZLE_SCHED_CTA && (tcgen05 || (!fp4 && batch > kCtaMaxBatch))) return PUZZLE_ERR_UNSUPPORTED;
  if (tcgen05 && desc->kv_dtype != PUZZLE_KV_FP8_E4M3) return PUZZLE_ERR_UNSUPPORTED;   // that kernel reads E4M3 codes only
  return PUZZLE_OK;
}

}  // namespace puzzle

using namespace puzzle;

extern "C" {

const char* puzzle_status_string(puzzle_status s) {
  switch (s) {
    case PUZZLE_OK: return "ok";
    case PUZZLE_ERR_NULL: return "a required pointer is NULL";
    case PUZZLE_ERR_SHAPE: return "inconsistent or out-of-range sizes";
    case PUZZLE_ERR_UNSUPPORTED: return "shape or dtype not supported by this build";
    case PUZZLE_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
    case PUZZLE_ERR_CUDA: return "a CUDA call or kernel launch failed";
  }
  return "unknown status";
}

int64_t puzzle_launch_count(void) { return g_launches.load(std::memory_order_relaxed); }

const char* puzzle_decode_attn_kernel_name(const puzzle_layer_desc* desc, const puzzle_kv_view* kv, int32_t batch,
                                           int32_t num_splits) {
  if (check_desc(desc) != PUZZLE_OK || !kv || batch <= 0 || batch > kMaxBatch || num_splits < PUZZLE_SCHED_WARP)
    return "invalid arguments";
  switch (pick_kernel(desc, kv, batch, num_splits)) {
    case Kernel::kCta: return "decode_attn_cta_kernel";
    case Kernel::kSmall: return "decode_attn_small_kernel";
    case Kernel::kGroup:
    case Kernel::kGroupCut: return "decode_attn_group_kernel";
    default: return "decode_attn_kernel";
  }
}

puzzle_status puzzle_kv_append(const puzzle_layer_desc* desc, const puzzle_kv_view* kv, const void* k_new,
                               const void* v_new, int32_t batch, int32_t* dev_status, void* stream) {
  puzzle_status st = check_desc(desc);
  if (st != PUZZLE_OK) return st;
  st = check_view(desc, kv, batch);
  if (st != PUZZLE_OK) return st;
  if (!k_new || !v_new) return PUZZLE_ERR_NULL;
  if (desc->kv_dtype == PUZZLE_KV_FP4_E2M1) {
    if (!aligned16(k_new) || !aligned16(v_new)) return PUZZLE_ERR_SHAPE;
    if (desc->num_kv_heads > kMaxAppendHeads) return PUZZLE_ERR_UNSUPPORTED;
    const cudaError_t e = append_fp4(desc, kv, k_new, v_new, nullptr, batch, 1, dev_status, static_cast<cudaStream_t>(stream));
    count_launch();
    return e == cudaSuccess ? PUZZLE_OK : PUZZLE_ERR_CUDA;
  }
  const long long threads = 2ll * batch * desc->num_kv_heads * (kHeadDim / 2);
  const int grid = (int)((threads + 255) / 256);
  const cudaError_t e = launch_dependent(
      kv_append_kernel, dim3(grid), dim3(256), 0, static_cast<cudaStream_t>(stream), kv->k_cache, kv->v_cache,
      static_cast<const __nv_bfloat16*>(k_new), static_cast<const __nv_bfloat16*>(v_new), kv->block_table,
      kv->seq_lens, kv->k_scale, kv->v_scale, kv->num_blocks, batch, desc->num_kv_heads, kv->max_blocks_per_seq,
      desc->kv_dtype, dev_status);
  count_launch();
  return e == cudaSuccess ? PUZZLE_OK : PUZZLE_ERR_CUDA;
}

puzzle_status puzzle_kv_append_tokens(const puzzle_layer_desc* desc, const puzzle_kv_view* kv, const void* k_new,
                                      const void* v_new, const int32_t* new_lens, int32_t batch, int32_t n_new,
                                      int32_t* dev_status, void* stream) {
  puzzle_status st = check_desc(desc);
  if (st != PUZZLE_OK) return st;
  st = check_view(desc, kv, batch);
  if (st != PUZZLE_OK) return st;
  if (!k_new || !v_new) return PUZZLE_ERR_NULL;
  if (n_new <= 0 || n_new > (1 << 20)) return PUZZLE_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(k_new) & 15) || (reinterpret_cast<uintptr_t>(v_new) & 15)) return PUZZLE_ERR_SHAPE;
  const long long per_seq = (long long)n_new * desc->num_kv_heads * (kHeadDim / 8);
  if (per_seq > 0x7fffffffll || batch > 65535) return PUZZLE_ERR_SHAPE;
  if (desc->kv_dtype == PUZZLE_KV_FP4_E2M1) {
    if (desc->num_kv_heads > kMaxAppendHeads) return PUZZLE_ERR_UNSUPPORTED;
    const cudaError_t e = append_fp4(desc, kv, k_new, v_new, new_lens, batch, n_new, dev_status,
                                     static_cast<cudaStream_t>(stream));
    count_launch();
    return e == cudaSuccess ? PUZZLE_OK : PUZZLE_ERR_CUDA;
  }
  const dim3 grid((unsigned)((per_seq + 255) / 256), (unsigned)batch, 2);
  const cudaError_t e = launch_dependent(
      kv_append_tokens_kernel, grid, dim3(256), 0, static_cast<cudaStream_t>(stream), kv->k_cache, kv->v_cache,
      static_cast<const uint4*>(k_new), static_cast<const uint4*>(v_new), new_lens, kv->block_table, kv->seq_lens,
      kv->k_scale, kv->v_scale, kv->num_blocks, batch, n_new, desc->num_kv_heads, kv->max_blocks_per_seq,
      desc->kv_dtype, dev_status);
  count_launch();
  return e == cudaSuccess ? PUZZLE_OK : PUZZLE_ERR_CUDA;
}

puzzle_status puzzle_kv_append_rope(const puzzle_layer_desc* desc, const puzzle_kv_view* kv, const puzzle_rope* rope,
                                    const puzzle_qkv* qkv, void* q_out, const int32_t* new_lens, int32_t batch,
                                    int32_t n_new, int32_t* dev_status, void* stream) {
  puzzle_status st = check_desc(desc);
  if (st != PUZZLE_OK) return st;
  st = check_view(desc, kv, batch);
  if (st != PUZZLE_OK) return st;
  if (!rope || !rope->cos_sin || !qkv || !qkv->k || !qkv->v || (qkv->q && !q_out)) return PUZZLE_ERR_NULL;
  if (n_new <= 0 || n_new > (1 << 20) || rope->num_positions <= 0) return PUZZLE_ERR_SHAPE;
  if (rope->rotary_dim <= 0 || rope->rotary_dim > desc->head_dim) return PUZZLE_ERR_SHAPE;
  if (rope->rotary_dim % 16) return PUZZLE_ERR_UNSUPPORTED;
  if (!aligned16(rope->cos_sin) || !aligned16(qkv->q) || !aligned16(qkv->k) || !aligned16(qkv->v) ||
      (qkv->q && !aligned16(q_out)))
    return PUZZLE_ERR_SHAPE;
  if (desc->num_kv_heads > kMaxAppendHeads) return PUZZLE_ERR_UNSUPPORTED;
  // rows are read 16 bytes at a time; the stride of a dimension of one means nothing
  const int64_t seq[3] = {qkv->k_seq_stride, qkv->v_seq_stride, qkv->q ? qkv->q_seq_stride : 0};
  const int64_t token[3] = {qkv->k_token_stride, qkv->v_token_stride, qkv->q ? qkv->q_token_stride : 0};
  for (int i = 0; i < 3; ++i)
    if ((batch > 1 && (seq[i] < 0 || seq[i] % 8)) || (n_new > 1 && (token[i] < 0 || token[i] % 8))) return PUZZLE_ERR_SHAPE;
  // in place: every row has to lie where its rotated form goes, or one row would overwrite another before it is read
  const int64_t row = (int64_t)desc->num_q_heads * desc->head_dim;
  if (qkv->q && q_out == qkv->q &&
      ((n_new > 1 && qkv->q_token_stride != row) || (batch > 1 && qkv->q_seq_stride != row * n_new)))
    return PUZZLE_ERR_SHAPE;
  AppendParams A = append_params(desc, kv, batch, n_new, new_lens, dev_status);
  A.q = static_cast<const __nv_bfloat16*>(qkv->q);
  A.k = static_cast<const __nv_bfloat16*>(qkv->k);
  A.v = static_cast<const __nv_bfloat16*>(qkv->v);
  A.q_seq_stride = qkv->q_seq_stride;
  A.q_token_stride = qkv->q_token_stride;
  A.k_seq_stride = qkv->k_seq_stride;
  A.k_token_stride = qkv->k_token_stride;
  A.v_seq_stride = qkv->v_seq_stride;
  A.v_token_stride = qkv->v_token_stride;
  A.q_out = static_cast<__nv_bfloat16*>(q_out);
  A.pos_offset = rope->pos_offset;
  A.cos_sin = rope->cos_sin;
  A.num_positions = rope->num_positions;
  A.rotary = rope->rotary_dim;
  const cudaError_t e =
      launch_append(A, desc->kv_dtype, true, rope->interleaved != 0, static_cast<cudaStream_t>(stream));
  count_launch();
  return e == cudaSuccess ? PUZZLE_OK : PUZZLE_ERR_CUDA;
}

puzzle_status puzzle_kv_read_tokens(const puzzle_layer_desc* desc, const puzzle_kv_view* kv, void* k_out, void* v_out,
                                    const int32_t* read_lens, int32_t batch, int32_t n_read, int32_t* dev_status,
                                    void* stream) {
  puzzle_status st = check_desc(desc);
  if (st != PUZZLE_OK) return st;
  st = check_view(desc, kv, batch);
  if (st != PUZZLE_OK) return st;
  if (!k_out || !v_out) return PUZZLE_ERR_NULL;
  if (desc->num_kv_heads > kMaxAppendHeads) return PUZZLE_ERR_UNSUPPORTED;
  if (n_read <= 0 || n_read > (1 << 24) || !aligned16(k_out) || !aligned16(v_out)) return PUZZLE_ERR_SHAPE;
  ReadParams R;
  std::memset(&R, 0, sizeof R);
  R.k_cache = kv->k_cache;
  R.v_cache = kv->v_cache;
  R.block_table = kv->block_table;
  R.seq_lens = kv->seq_lens;
  R.read_lens = read_lens;
  R.k_scale = kv->k_scale;
  R.v_scale = kv->v_scale;
  R.k_out = static_cast<__nv_bfloat16*>(k_out);
  R.v_out = static_cast<__nv_bfloat16*>(v_out);
  R.dev_status = dev_status;
  R.num_blocks = kv->num_blocks;
  R.batch = batch;
  R.n_read = n_read;
  R.Hkv = desc->num_kv_heads;
  R.max_blocks_per_seq = kv->max_blocks_per_seq;
  const cudaError_t e = launch_read_tokens(R, desc->kv_dtype, static_cast<cudaStream_t>(stream));
  count_launch();
  return e == cudaSuccess ? PUZZLE_OK : PUZZLE_ERR_CUDA;
}

size_t puzzle_decode_attn_workspace_bytes(const puzzle_layer_desc* desc, int32_t batch, int32_t num_splits) {
  if (check_desc(desc) != PUZZLE_OK || batch <= 0 || batch > kMaxBatch || num_splits < PUZZLE_SCHED_WARP) return 0;
  return counter_bytes(batch, desc->num_kv_heads) +
         workspace_floats(batch, desc->num_kv_heads, num_splits > 0 ? num_splits : 0, desc->kv_dtype) * sizeof(float) +
         pair_parts_bytes((size_t)batch * desc->num_kv_heads, desc->kv_dtype);
}

static puzzle_status decode_attn_impl(const puzzle_layer_desc* desc, const puzzle_kv_view* kv, const void* q,
                                      const float* sinks, void* out, float* lse_out, int32_t batch,
                                      int32_t num_splits, void* workspace, size_t workspace_bytes,
                                      int32_t* dev_status, void* stream, bool tcgen05, bool out_f32 = false) {
  puzzle_status st = check_decode_attn_args(desc, kv, q, out, batch, num_splits, tcgen05);
  if (st != PUZZLE_OK) return st;
  const int Hkv = desc->num_kv_heads;
  const size_t cbytes = counter_bytes(batch, Hkv);
  const int splits = num_splits > 0 ? num_splits : 0;   // the kernels know explicit splits (S) and balanced (0)
  const size_t pfloats = workspace_floats(batch, Hkv, splits, desc->kv_dtype);
  const size_t need = cbytes + pfloats * sizeof(float) + pair_parts_bytes((size_t)batch * Hkv, desc->kv_dtype);
  if (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15)) return PUZZLE_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);

  const int ctas = grid_ctas();
  const size_t rows = pfloats / (kHeadDim + 1);
  float* part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) + cbytes);
  float* part_lse = part_o + rows * kHeadDim;

  DecodeParams P;
  std::memset(&P, 0, sizeof P);
  const bool tc = tcgen05;
  if (!set_cache(&P, desc, kv, tc ? 64 : 128)) return PUZZLE_ERR_CUDA;
  P.q = static_cast<const __nv_bfloat16*>(q);
  P.block_table = kv->block_table;
  P.seq_lens = kv->seq_lens;
  P.k_scale = kv->k_scale;
  P.v_scale = kv->v_scale;
  P.part_o = part_o;
  P.part_lse = part_lse;
  P.cta_words = static_cast<int32_t*>(workspace);
  P.counters = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + cta_word_bytes());
  P.sinks = sinks;
  P.out = out_f32 ? nullptr : static_cast<__nv_bfloat16*>(out);
  P.out_f32 = out_f32 ? static_cast<float*>(out) : nullptr;
  P.lse_out = lse_out;
  P.dev_status = dev_status;
  P.num_blocks = kv->num_blocks;
  P.batch = batch;
  P.Hkv = Hkv;
  P.max_blocks_per_seq = kv->max_blocks_per_seq;
  P.window = desc->window;
  P.num_splits = splits;
  P.sm_scale_log2e = desc->sm_scale * 1.4426950408889634f;

  cudaError_t le;
  if (tc) {
    le = launch_decode_attn_tc(P, ctas, s, &device_info().smem_tc);
  } else {
    switch (pick_kernel(desc, kv, batch, num_splits)) {
      case Kernel::kGroup:
      case Kernel::kGroupCut: {
        const bool cut = pick_kernel(desc, kv, batch, num_splits) == Kernel::kGroupCut;
        P.pair_parts = reinterpret_cast<int2*>(part_lse + rows);
        le = launch_decode_attn_group(P, group_warps(tiles_per_pair_bound(desc, kv), (long long)batch * Hkv, cut), cut, ctas, s,
                                      device_info().smem_group);
        break;
      }
      case Kernel::kCta:
        le = launch_decode_attn_cta(P, desc->kv_dtype == PUZZLE_KV_FP8_E4M3, ctas, s, device_info().smem_cta);
        break;
      case Kernel::kSmall:
        le = launch_decode_attn_small(P, desc->kv_dtype, ctas, s, device_info().smem_small);
        break;
      case Kernel::kWarpWholePairs:
        P.num_splits = 1;
        le = launch_decode_attn(P, desc->kv_dtype, ctas, s, device_info().smem_warp);
        break;
      default:
        le = launch_decode_attn(P, desc->kv_dtype, ctas, s, device_info().smem_warp);
    }
  }
  if (le != cudaSuccess) return PUZZLE_ERR_CUDA;
  count_launch();

  return PUZZLE_OK;
}

puzzle_status puzzle_decode_attn(const puzzle_layer_desc* desc, const puzzle_kv_view* kv, const void* q,
                                 const float* sinks, void* out, float* lse_out, int32_t batch, int32_t num_splits,
                                 void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
  return decode_attn_impl(desc, kv, q, sinks, out, lse_out, batch, num_splits, workspace, workspace_bytes, dev_status,
                          stream, false);
}

puzzle_status puzzle_decode_attn_tcgen05(const puzzle_layer_desc* desc, const puzzle_kv_view* kv, const void* q,
                                         const float* sinks, void* out, float* lse_out, int32_t batch,
                                         int32_t num_splits, void* workspace, size_t workspace_bytes,
                                         int32_t* dev_status, void* stream) {
  return decode_attn_impl(desc, kv, q, sinks, out, lse_out, batch, num_splits, workspace, workspace_bytes, dev_status,
                          stream, true);
}

// Device staging of one step whose inputs and result live in host memory: q, k_new, v_new, out, each padded to 256 bytes.
static size_t staging_part(size_t elems) { return (elems * sizeof(__nv_bfloat16) + 255) & ~(size_t)255; }

size_t puzzle_decode_step_host_staging_bytes(const puzzle_layer_desc* desc, int32_t batch) {
  if (check_desc(desc) != PUZZLE_OK || batch <= 0 || batch > kMaxBatch) return 0;
  const size_t qn = (size_t)batch * desc->num_q_heads * desc->head_dim, kn = (size_t)batch * desc->num_kv_heads * desc->head_dim;
  return 2 * staging_part(qn) + 2 * staging_part(kn);
}

puzzle_status puzzle_decode_step_host(const puzzle_layer_desc* desc, const puzzle_kv_view* kv, const void* q_host,
                                      const void* k_new_host, const void* v_new_host, const float* sinks,
                                      void* out_host, int32_t batch, int32_t num_splits, void* staging,
                                      size_t staging_bytes, void* workspace, size_t workspace_bytes,
                                      int32_t* dev_status, void* stream) {
  if (!q_host || !k_new_host || !v_new_host || !out_host) return PUZZLE_ERR_NULL;
  const size_t need = puzzle_decode_step_host_staging_bytes(desc, batch);
  if (need == 0) return check_desc(desc) != PUZZLE_OK ? check_desc(desc) : PUZZLE_ERR_SHAPE;
  if (!staging || staging_bytes < need || (reinterpret_cast<uintptr_t>(staging) & 255)) return PUZZLE_ERR_WORKSPACE;
  const size_t qn = (size_t)batch * desc->num_q_heads * desc->head_dim, kn = (size_t)batch * desc->num_kv_heads * desc->head_dim;
  char* dq = static_cast<char*>(staging);
  char* dk = dq + staging_part(qn);
  char* dv = dk + staging_part(kn);
  char* dout = dv + staging_part(kn);
  // every host-visible error of the two device calls is found before the first copy is enqueued
  puzzle_status st = check_decode_attn_args(desc, kv, dq, dout, batch, num_splits, false);
  if (st != PUZZLE_OK) return st;
  if (desc->kv_dtype == PUZZLE_KV_FP4_E2M1 && desc->num_kv_heads > kMaxAppendHeads) return PUZZLE_ERR_UNSUPPORTED;
  if (!workspace || workspace_bytes < puzzle_decode_attn_workspace_bytes(desc, batch, num_splits) ||
      (reinterpret_cast<uintptr_t>(workspace) & 15))
    return PUZZLE_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const size_t qb = qn * sizeof(__nv_bfloat16), kb = kn * sizeof(__nv_bfloat16);
  const char* hq = static_cast<const char*>(q_host);
  if (static_cast<const char*>(k_new_host) == hq + qb && static_cast<const char*>(v_new_host) == hq + qb + kb &&
      qb % 256 == 0 && kb % 256 == 0 && one_pinned_range(hq, qb + 2 * kb)) {
    // the three inputs follow each other in one pinned buffer as they do in the staging area: one copy
    if (cudaMemcpyAsync(dq, q_host, qb + 2 * kb, cudaMemcpyHostToDevice, s) != cudaSuccess) return PUZZLE_ERR_CUDA;
  } else if (cudaMemcpyAsync(dq, q_host, qb, cudaMemcpyHostToDevice, s) != cudaSuccess ||
             cudaMemcpyAsync(dk, k_new_host, kb, cudaMemcpyHostToDevice, s) != cudaSuccess ||
             cudaMemcpyAsync(dv, v_new_host, kb, cudaMemcpyHostToDevice, s) != cudaSuccess) {
    return PUZZLE_ERR_CUDA;
  }
  st = puzzle_kv_append(desc, kv, dk, dv, batch, dev_status, stream);
  if (st != PUZZLE_OK) return st;
  st = puzzle_decode_attn(desc, kv, dq, sinks, dout, nullptr, batch, num_splits, workspace, workspace_bytes, dev_status,
                          stream);
  if (st != PUZZLE_OK) return st;
  return cudaMemcpyAsync(out_host, dout, qn * sizeof(__nv_bfloat16), cudaMemcpyDeviceToHost, s) == cudaSuccess
             ? PUZZLE_OK
             : PUZZLE_ERR_CUDA;
}

puzzle_status puzzle_decode_attn_partial(const puzzle_layer_desc* desc, const puzzle_kv_view* kv, const void* q,
                                         float* o_part, float* lse_part, int32_t batch, int32_t num_splits,
                                         void* workspace, size_t workspace_bytes, int32_t* dev_status,
                                         void* stream) {
  if (!lse_part) return PUZZLE_ERR_NULL;
  return decode_attn_impl(desc, kv, q, nullptr, o_part, lse_part, batch, num_splits, workspace, workspace_bytes,
                          dev_status, stream, false, true);
}

// Room for the largest supported batch * ceil(n_q / 2) whatever the call's own, for the same reason as counter_bytes.
static size_t tokens_counter_bytes(int batch, int n_q, int Hkv) {
  const size_t n = std::max<size_t>(decode_attn_tokens_counters(batch, n_q, Hkv), (size_t)kTokMaxRows * Hkv);
  return (n * sizeof(int32_t) + 255) & ~(size_t)255;
}

size_t puzzle_decode_attn_tokens_workspace_bytes(const puzzle_layer_desc* desc, int32_t batch, int32_t n_q) {
  if (check_desc(desc) != PUZZLE_OK || batch <= 0 || n_q <= 0 || (long long)batch * ((n_q + 1) / 2) > kTokMaxRows)
    return 0;
  return tokens_counter_bytes(batch, n_q, desc->num_kv_heads) +
         decode_attn_tokens_partial_rows(grid_ctas(), batch, n_q, desc->num_kv_heads) * (kHeadDim + 1) * sizeof(float) +
         pair_parts_bytes((size_t)batch * ((n_q + 1) / 2) * desc->num_kv_heads, desc->kv_dtype);
}

puzzle_status puzzle_decode_attn_tokens_workspace_init(const puzzle_layer_desc* desc, int32_t batch, int32_t n_q,
                                                       void* workspace, size_t workspace_bytes, void* stream) {
  puzzle_status st = check_desc(desc);
  if (st != PUZZLE_OK) return st;
  if (batch <= 0 || n_q <= 0 || (long long)batch * ((n_q + 1) / 2) > kTokMaxRows) return PUZZLE_ERR_SHAPE;
  const size_t cbytes = tokens_counter_bytes(batch, n_q, desc->num_kv_heads);
  if (!workspace || workspace_bytes < cbytes || (reinterpret_cast<uintptr_t>(workspace) & 15))
    return PUZZLE_ERR_WORKSPACE;
  return cudaMemsetAsync(workspace, 0, cbytes, static_cast<cudaStream_t>(stream)) == cudaSuccess ? PUZZLE_OK
                                                                                                  : PUZZLE_ERR_CUDA;
}

puzzle_status puzzle_decode_attn_tokens(const puzzle_layer_desc* desc, const puzzle_kv_view* kv, const void* q,
                                        const int32_t* q_lens, const float* sinks, void* out, float* lse_out,
                                        int32_t batch, int32_t n_q, void* workspace, size_t workspace_bytes,
                                        int32_t* dev_status, void* stream) {
  puzzle_status st = check_decode_attn_args(desc, kv, q, out, batch, 0, false);
  if (st != PUZZLE_OK) return st;
  if (n_q <= 0 || (long long)batch * ((n_q + 1) / 2) > kTokMaxRows) return PUZZLE_ERR_SHAPE;
  if (desc->kv_dtype == PUZZLE_KV_BF16) return PUZZLE_ERR_UNSUPPORTED;   // the bf16 cache goes one row per token
  const int Hkv = desc->num_kv_heads;
  const size_t need = puzzle_decode_attn_tokens_workspace_bytes(desc, batch, n_q);
  if (!workspace || workspace_bytes < need || (reinterpret_cast<uintptr_t>(workspace) & 15)) return PUZZLE_ERR_WORKSPACE;
  const size_t cbytes = tokens_counter_bytes(batch, n_q, Hkv);
  const size_t rows = decode_attn_tokens_partial_rows(grid_ctas(), batch, n_q, Hkv);
  DecodeParams P;
  std::memset(&P, 0, sizeof P);
  if (!set_cache(&P, desc, kv, 128)) return PUZZLE_ERR_CUDA;
  P.q = static_cast<const __nv_bfloat16*>(q);
  P.block_table = kv->block_table;
  P.seq_lens = kv->seq_lens;
  P.k_scale = kv->k_scale;
  P.v_scale = kv->v_scale;
  P.part_o = reinterpret_cast<float*>(static_cast<char*>(workspace) + cbytes);
  P.part_lse = P.part_o + rows * kHeadDim;
  P.counters = static_cast<int32_t*>(workspace);
  P.sinks = sinks;
  P.out = static_cast<__nv_bfloat16*>(out);
  P.lse_out = lse_out;
  P.dev_status = dev_status;
  P.num_blocks = kv->num_blocks;
  P.batch = batch;
  P.Hkv = Hkv;
  P.max_blocks_per_seq = kv->max_blocks_per_seq;
  P.window = desc->window;
  P.n_q = n_q;
  P.q_lens = q_lens;
  P.sm_scale_log2e = desc->sm_scale * 1.4426950408889634f;
  const int ctas = grid_ctas();
  cudaStream_t cs = static_cast<cudaStream_t>(stream);
  cudaError_t le;
  if (desc->kv_dtype == PUZZLE_KV_FP4_E2M1) {
    const long long tiles = tiles_per_pair_bound(desc, kv), pairs = (long long)batch * ((n_q + 1) / 2) * Hkv;
    const bool cut = !whole_pairs_tokens(tiles, pairs);
    P.pair_parts = reinterpret_cast<int2*>(P.part_lse + rows);
    le = launch_decode_attn_tokens_group(P, tokens_group_warps(tiles, pairs, cut), cut, ctas, cs,
                                         device_info().smem_tokens_group);
  } else {
    le = launch_decode_attn_tokens(P, ctas, cs, &device_info().smem_tokens);
  }
  if (le != cudaSuccess) return PUZZLE_ERR_CUDA;
  count_launch();
  return PUZZLE_OK;
}

puzzle_status puzzle_decode_attn_workspace_init(const puzzle_layer_desc* desc, int32_t batch, void* workspace,
                                                size_t workspace_bytes, void* stream) {
  puzzle_status st = check_desc(desc);
  if (st != PUZZLE_OK) return st;
  if (batch <= 0 || batch > kMaxBatch) return PUZZLE_ERR_SHAPE;
  const size_t cbytes = counter_bytes(batch, desc->num_kv_heads);
  if (!workspace || workspace_bytes < cbytes || (reinterpret_cast<uintptr_t>(workspace) & 15))
    return PUZZLE_ERR_WORKSPACE;
  return cudaMemsetAsync(workspace, 0, cbytes, static_cast<cudaStream_t>(stream)) == cudaSuccess ? PUZZLE_OK
                                                                                                  : PUZZLE_ERR_CUDA;
}

puzzle_status puzzle_kv_amax_update(const void* x, int64_t n_tokens, int32_t num_kv_heads, int32_t head_dim,
                                    float* amax, void* stream) {
  if (!amax || (!x && n_tokens > 0)) return PUZZLE_ERR_NULL;
  if (n_tokens < 0 || num_kv_heads <= 0 || num_kv_heads > calibrate_max_heads() || head_dim <= 0 || head_dim % 8)
    return PUZZLE_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(x) & 15) || (reinterpret_cast<uintptr_t>(amax) & 3)) return PUZZLE_ERR_SHAPE;
  if (n_tokens == 0) return PUZZLE_OK;
  if (launch_amax_update(x, n_tokens, num_kv_heads, head_dim, amax, grid_ctas(), static_cast<cudaStream_t>(stream)) !=
      cudaSuccess)
    return PUZZLE_ERR_CUDA;
  count_launch();
  return PUZZLE_OK;
}

puzzle_status puzzle_kv_scales_from_amax(const float* amax, int32_t num_kv_heads, int32_t pow2, float* scale_out,
                                         void* stream) {
  if (!amax || !scale_out) return PUZZLE_ERR_NULL;
  if (num_kv_heads <= 0 || num_kv_heads > calibrate_max_heads()) return PUZZLE_ERR_SHAPE;
  if (launch_scales_from_amax(amax, num_kv_heads, pow2, scale_out, static_cast<cudaStream_t>(stream)) != cudaSuccess)
    return PUZZLE_ERR_CUDA;
  count_launch();
  return PUZZLE_OK;
}

puzzle_status puzzle_attn_merge_strided(const float* part_o, const float* part_lse, int64_t o_row_stride,
                                        int64_t o_part_stride, int64_t lse_row_stride, int64_t lse_part_stride,
                                        const int32_t* num_parts, const float* sinks, void* out, float* lse_out,
                                        int32_t batch, int32_t Hq, int32_t D, int32_t S, void* stream) {
  if (!part_o || !part_lse || !out) return PUZZLE_ERR_NULL;
  if (batch <= 0 || Hq <= 0 || S <= 0 || D <= 0) return PUZZLE_ERR_SHAPE;
  if (D % 64 != 0 || D > 512) return PUZZLE_ERR_UNSUPPORTED;
  if ((reinterpret_cast<uintptr_t>(part_o) & 7) || (reinterpret_cast<uintptr_t>(out) & 3)) return PUZZLE_ERR_SHAPE;
  if (o_row_stride < 0 || o_part_stride < 0 || lse_row_stride < 0 || lse_part_stride < 0 || (o_row_stride & 1) ||
      (o_part_stride & 1))
    return PUZZLE_ERR_SHAPE;   // partial rows are read two floats at a time
  MergeParams M;
  std::memset(&M, 0, sizeof M);
  M.part_o = part_o;
  M.part_lse = part_lse;
  M.o_row_stride = o_row_stride;
  M.o_part_stride = o_part_stride;
  M.lse_row_stride = lse_row_stride;
  M.lse_part_stride = lse_part_stride;
  M.num_parts = num_parts;
  M.sinks = sinks;
  M.out = static_cast<__nv_bfloat16*>(out);
  M.lse_out = lse_out;
  M.batch = batch;
  M.Hq = Hq;
  M.D = D;
  M.S = S;
  const long long rows = (long long)batch * Hq;
  attn_merge_kernel<<<(unsigned)((rows + kWarps - 1) / kWarps), kWarps * 32, 0, static_cast<cudaStream_t>(stream)>>>(M);
  count_launch();
  return cudaGetLastError() == cudaSuccess ? PUZZLE_OK : PUZZLE_ERR_CUDA;
}

puzzle_status puzzle_attn_merge(const float* part_o, const float* part_lse, const int32_t* num_parts,
                                const float* sinks, void* out, float* lse_out, int32_t batch, int32_t Hq, int32_t D,
                                int32_t S, void* stream) {
  return puzzle_attn_merge_strided(part_o, part_lse, (int64_t)S * D, D, S, 1, num_parts, sinks, out, lse_out, batch, Hq,
                                   D, S, stream);
}

puzzle_status puzzle_hbm_read_probe(const void* buf, size_t bytes, uint64_t* sink, void* stream) {
  if (!buf || !sink) return PUZZLE_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(buf) & 15) || (bytes & 15) || bytes == 0) return PUZZLE_ERR_SHAPE;
  const int ctas = grid_ctas() * 4;
  hbm_read_probe_kernel<<<ctas, 512, 0, static_cast<cudaStream_t>(stream)>>>(
      static_cast<const uint4*>(buf), bytes / 16, reinterpret_cast<unsigned long long*>(sink));
  count_launch();
  return cudaGetLastError() == cudaSuccess ? PUZZLE_OK : PUZZLE_ERR_CUDA;
}

}  // extern "C"
