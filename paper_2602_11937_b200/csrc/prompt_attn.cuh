// Attention of many query tokens per sequence (whole prompts, chunks over the cache): parameters and launch.
#pragma once

#include <cuda.h>

#include "common.cuh"

namespace puzzle {

// Where keys and values come from.
enum PromptSource { kSrcPacked = 0, kSrcBf16 = 1, kSrcFp8 = 2, kSrcFp4 = 3 };

struct PromptParams {
  CUtensorMap tmQ;            // [total][Hq][64] bf16, box = 16 tokens of one KV head's 8 query heads
  CUtensorMap tmK, tmV;       // packed keys and values [total][Hkv][64]: box = 128 tokens of one head (kSrcPacked only)
  const void *k_cache, *v_cache;
  const __nv_bfloat16* v;     // packed values
  long long v_token_stride;   // in elements
  const int32_t *block_table, *seq_lens, *starts;
  const float *k_scale, *v_scale, *sinks;
  __nv_bfloat16* out;
  float *lse_out, *part_o, *part_lse;
  int32_t* dev_status;
  long long num_blocks;
  int batch, total, Hkv, max_blocks_per_seq, window, splits, turns;
  float sm_scale_log2e;
};

// splits: parts that the keys of a group of tokens are cut into (1: the kernel writes the output, else partials that a second
// kernel merges).  turns: streams to a tile of rows; a group is 64 / turns tokens.
struct PromptPlan {
  int splits, turns;
};
// fetch: what bringing a tile of 128 keys in costs, in steps of 64 keys.
PromptPlan prompt_plan(int batch, int total, int Hkv, long long key_bound, bool may_split, double fetch, int sm_count);
int prompt_most_splits(int batch, int total, int Hkv, int sm_count);
size_t prompt_partial_bytes(int total, int Hkv, int splits);
cudaError_t launch_prompt_attn(const PromptParams& P, PromptSource src, cudaStream_t s, int* smem_limit);

}  // namespace puzzle
