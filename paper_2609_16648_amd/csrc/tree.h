// Internal interfaces of the draft-tree operators: append, masks, attention, accept, commit.
#pragma once

#include "forward.h"

namespace gm {

constexpr int kMaxNodes = 64;      // nodes of a tree: one bit each in a mask, one lane each in a wave
// sequences and rows per call: a workgroup's 256 threads times their number stay below 2^32 per launch
constexpr int kMaxTrees = 1 << 22, kMaxAppendRows = 1 << 27;

struct AppendArgs {
  int dtype, B, T, n_heads, n_kv, head_dim;   // n_heads 0: no queries
  int page_size, max_pages, num_pages;
  const int32_t *row_start, *offsets;         // or null (see gm_kv_append)
  const int32_t *block_table, *seq_lens;
  const void *q, *k, *v;
  long q_stride, k_stride, v_stride;          // elements between rows
  const void *q_norm, *k_norm;                // or null
  void *q_out, *k_pages, *v_pages;
  double log2_base;                           // of rope_base
  float eps;
  int32_t *dev_err;
};
void launch_kv_append(const AppendArgs &a, hipStream_t s);

void launch_tree_masks(int B, int N, const int32_t *parents, const int32_t *n_nodes, uint64_t *masks, int32_t *depths,
                       int32_t *dev_err, hipStream_t s);
void launch_tree_accept(int B, int N, const int32_t *parents, const int32_t *tokens, const int32_t *next_ids,
                        const int32_t *n_nodes, int32_t *path, int32_t *n_accept, int32_t *out_tokens, hipStream_t s);
void launch_tree_commit(const gm_model_config &cfg, const gm_kv_cache &c, int B, int N, const int32_t *path,
                        const int32_t *n_accept, int32_t *slots, int32_t *dev_err, hipStream_t s);

// attention of N tree nodes per sequence (attention.hip): a.R is N, a.blk_len the nodes per sequence or null
AttnPlan plan_tree_attention(const gm_model_config &cfg, int B, int N);
void run_tree_attention(const AttnArgs &a, const uint64_t *masks, const AttnPlan &p, char *ws, hipStream_t s);

}  // namespace gm
