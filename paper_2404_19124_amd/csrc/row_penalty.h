// What changes the logits of a token tree's rows, token by token.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_utils.h"
#include "rows_internal.h"

namespace specdraft {

// eight neighbours; rows of an odd length start anywhere, so their words are not aligned to 16 bytes (the compiler's memcpy is one
// 16-byte load all the same)
template <typename T>
__device__ __forceinline__ T load_words(const void* from) {
  T x;
  __builtin_memcpy(&x, from, sizeof(T));
  return x;
}

__device__ __forceinline__ float to_f32(uint16_t x) { return bf16_bits_to_f32(x); }
__device__ __forceinline__ float to_f32(float x) { return x; }

// What changes one sequence's logits (row by row: allowed).
struct RowPenalty {
  const int32_t* counts;
  const uint32_t *seen, *allowed;
  const float* bias;
  float rep, pres, freq;
};

// A token by the whole formula; c: its occurrences.
__device__ __forceinline__ float penalized(float v, int c, bool bit, float bias, bool allowed, const RowPenalty& pen) {
// (a product and a difference are rounded one by one: what is chosen must not hang on the compiler's choice)
#pragma clang fp contract(off)
  if (bit || c > 0) v = v > 0.0f ? v / pen.rep : v * pen.rep;
  v = v - pen.freq * (float)c;
  if (c > 0) v = v - pen.pres;
  if (pen.bias) v = v + bias;
  return allowed ? v : SPEC_NEG_INF;
}

// of sequence q's row `row` of all
__device__ __forceinline__ RowPenalty penalty_of(const spec_penalties_t& p, int q, int row, int V) {
  const int n_words = (V + 31) / 32;
  RowPenalty pen;
  pen.counts = p.counts ? p.counts + (int64_t)q * V : nullptr;
  pen.seen = p.seen ? p.seen + (int64_t)q * n_words : nullptr;
  const int mask_row = p.allowed ? p.mask_row[row] : -1, bias_row = p.bias ? p.bias_row[q] : -1;
  pen.bias = bias_row >= 0 && bias_row < p.n_bias ? p.bias + (int64_t)bias_row * V : nullptr;
  pen.allowed = mask_row >= 0 && mask_row < p.n_allowed ? p.allowed + (int64_t)mask_row * n_words : nullptr;
  pen.rep = p.repetition ? p.repetition[q] : 1.0f, pen.pres = p.presence ? p.presence[q] : 0.0f;
  pen.freq = p.frequency ? p.frequency[q] : 0.0f;
  return pen;
}

}  // namespace specdraft
