// Internal declarations of the operators on the rows of a token tree (attention, cache, logits).
// Not part of the public boundary (that is include/spec.h).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/spec.h"

namespace specdraft {

constexpr int64_t kMaxSlots = 1 << 30;   // tokens of a cache, of a block table's row, of a slot map

constexpr int kMaxHeadEntries = 1 << 25;   // rows, or entries, of one call on rows of heads (a launch has fewer than 2^32 threads)

constexpr int kMaxLogitsRows = (1 << 23) - 8;   // rows of one call on logits
constexpr int kMaxSampledRows = 1 << 20, kMaxSampledBatch = 1 << 17;   // of one whose tokens are drawn

// ---- attention of the rows over a paged cache and their own ancestors ----------------
struct AttentionJob {
  const void *q, *k_new, *v_new, *k, *v;
  void* out;
  // strides in bytes: of sequences, rows and heads (q, new, out); of blocks, slots and heads (cache)
  int64_t q_seq, q_row, q_head, new_seq, new_row, new_head, out_seq, out_row, out_head;
  int64_t block, slot, cache_head;
  const int32_t *block_table, *ctx_len, *node_parent, *n_nodes;
  int batch, M, q_heads, kv_heads, head_dim;
  int max_blocks, n_blocks, block_size;
  int offsets_fit; // every key lies within 4 GiB of its head's first one, in the cache and among the rows
  int one_place;   // 16 tokens from a multiple of 16 on lie in one block, at offsets of 31 bits
  const uint8_t *k_scale, *v_scale;               // of a cache of four bits, whose strides above are its codes'
  int64_t scale_block, scale_slot, scale_head;
  float scale;
  void* workspace;
};
int64_t attention_workspace(int batch, int M, int q_heads, int kv_heads, int head_dim, bool bf16);
hipError_t launch_attention(const AttentionJob& job, bool bf16, hipStream_t st);
hipError_t launch_packed_attention(const AttentionJob& job, hipStream_t st);   // workspace: attention_workspace's of bfloat16

// ---- block tables and slot maps --------------------------------------------------------
struct ExtendJob {
  const int32_t *ctx_len, *add;
  int32_t *new_len, *added;
  int batch;
  int32_t* block_table;
  int max_blocks;
  int32_t* ring;
  int n_blocks;
  const int32_t* ring_state;
  int32_t* ring_state_new;
  int block_size;
  int32_t *row_start, *slot, *pos, *src_row;
  int cap;
  const int32_t* path_row;
  int path_width, seq_rows;
};
hipError_t launch_extend(const ExtendJob& job, hipStream_t st);

// ---- keys and values into their slots ----------------------------------------------------
struct StoreJob {
  const uint8_t *k_new, *v_new;
  uint8_t *k, *v;
  // strides in bytes
  int64_t new_layer, new_row, new_head, layer, block, slot_stride, head;
  int layers, rows, kv_heads, row_words;   // 16-byte words of one head's row
  int n_slots, block_size;
  const int32_t *slot, *src_row;
  int count;
};
hipError_t launch_store(const StoreJob& job, hipStream_t st);

// ---- rows of heads: norm, rotation, and into a cache -------------------------------------
// Rows that one launch reads and writes: the queries and the keys, or the keys and the values.
struct HeadSide {
  const uint8_t* from;
  uint8_t* to;
  // strides in bytes; far: of sequences, or of layers; to_row: of rows, or of slots
  int64_t from_far, from_row, from_head, to_far, to_block, to_row, to_head;
  const float* weight;   // of the norm, or NULL
  int heads;
  bool turned;
};
struct HeadsJob {
  HeadSide side[2];
  int entries, layers, row_words, head_dim;   // 16-byte words of one head's row
  // rotation: NULL: none; half_words: words of the first elements of the pairs
  const float *cos, *sin;
  int n_pos, half_words, pairs;
  double eps;
  const int32_t* pos;
  // rows of trees: entry q * (M + 1) + r
  int M;
  const int32_t *ctx_len, *node_depth, *n_nodes;
  // into a cache: entry t
  const int32_t *slot, *src_row;
  int rows, n_slots, block_size;
  int lanes, trips;      // (the launch's)
};
hipError_t launch_heads(HeadsJob job, bool bf16, bool append, hipStream_t st);

// ---- a cache of four bits ------------------------------------------------------------------
struct PackJob {
  const uint8_t *k_new, *v_new;
  uint8_t *k, *v, *k_scale, *v_scale;
  // strides in bytes
  int64_t new_layer, new_row, new_head, layer, block, slot_stride, head, scale_layer, scale_block, scale_slot, scale_head;
  int entries, layers, rows, heads, groups;   // groups of 32 elements of a head
  const float *cos, *sin, *weight;
  int n_pos, half_words, pairs;
  double eps;
  const int32_t *pos, *slot, *src_row;
  int n_slots, block_size;
  int lanes, trips;      // (the launch's)
};
hipError_t launch_pack(PackJob job, hipStream_t st);

struct UnpackJob {
  const uint8_t *k, *v, *k_scale, *v_scale;
  uint8_t *k_out, *v_out;
  int64_t layer, block, slot_stride, head, scale_layer, scale_block, scale_slot, scale_head, out_layer, out_row, out_head;
  int count, layers, heads, groups;
  const int32_t* slot;
  int n_slots, block_size;
};
hipError_t launch_unpack(const UnpackJob& job, hipStream_t st);

// ---- logits of the rows -------------------------------------------------------------------
struct LogitsJob {
  const void* logits;
  int batch, M, V;
  spec_penalties_t pen;                    // all NULL: plain logits
  const int32_t *node_tok, *node_parent, *n_nodes;
  void* out;                               // processed logits, or
  int32_t* greedy;                         // their first maximum per row
};
hipError_t launch_logits(const LogitsJob& job, bool bf16, hipStream_t st);

struct AcceptTreeJob {
  const int32_t *greedy, *cand, *cand_node, *n_cand, *n_nodes;
  int batch, M, B, n, V;
  int32_t *accept_len, *best_cand, *out_tokens, *n_out, *path_row, *accept_all, *counts;
  uint32_t* seen;
};
hipError_t launch_accept_tree(const AcceptTreeJob& job, hipStream_t st);

// ---- verification against the target's probabilities ---------------------------------------
struct SamplePart {        // of some of a row's tokens
  float top;               // the largest processed logit
  int32_t first;           // its first token, without a temperature
  double sum;              // of the weights relative to it
};
struct SampleSlot {        // where a sequence's path has led
  int32_t done, level, row, unused;
  int32_t tok[SPEC_MAX_STAGES], path[SPEC_MAX_STAGES];
  double weight[SPEC_MAX_STAGES], sum[SPEC_MAX_STAGES];   // the tokens' and their rows'
};
struct SampleJob {
  const void* logits;
  int batch, M, V, n;
  spec_penalties_t pen;
  int paths;               // whether a row's path counts
  const int32_t *node_tok, *node_parent, *n_nodes;
  const float *temperature, *uniform;
  int32_t *accept_len, *out_tokens, *n_out, *path_row;
  float* out_logp;
  int32_t* counts;
  uint32_t* seen;
  // (the launch's)
  int parts, span, run, all_rows;
  SamplePart* part;        // of all rows, or of two rows of every sequence
  float* node_v;
  SampleSlot* slot;
};
int64_t sample_workspace(int batch, int M, int V);
hipError_t launch_sample(SampleJob job, void* workspace, bool bf16, hipStream_t st);

}  // namespace specdraft
