// Internal declarations of the operators on the rows of a token tree (attention, cache, logits).
// Not part of the public boundary (that is include/spec.h).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/spec.h"

namespace specdraft {

constexpr int64_t kMaxSlots = 1 << 30;   // tokens of a cache, of a block table's row, of a slot map

constexpr int kMaxLogitsRows = (1 << 23) - 8;   // rows of one call on logits

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
  float scale;
  void* workspace;
};
int64_t attention_workspace(int batch, int M, int q_heads, int kv_heads, int head_dim, bool bf16);
hipError_t launch_attention(const AttentionJob& job, bool bf16, hipStream_t st);

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

}  // namespace specdraft
