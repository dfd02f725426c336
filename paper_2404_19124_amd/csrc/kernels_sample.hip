// Verification of a token tree against the base model's probabilities, from given random numbers.
//   v_t: a row's processed logits (row_penalty.h);  w_t = exp((v_t - max v) / temperature);  S = sum of all w
// A row's mass S lies on a line: first the drafted tokens of the row, in the order of their nodes, then all others by number.  The token at
// u * S is the row's token, u being the sequence's random number for that depth: with a drafted one the path goes down to its node, with
// another it ends, and that token is the last one emitted.  Every token so has its probability, whatever was drafted.
//
// Weights and sums are 64-bit numbers: where an end of a token's stretch lies is off by some 1e-13 of S, so that the choice among 130000
// tokens hangs on the order of sums once in 1e8 calls (with float32 weights, 1e-7 each: once in a hundred).  A product in 64 bits costs
// as much here as one in float32.
//
// A row is taken by `parts` workgroups, PARTIALS of which (largest, sum relative to it) are joined by whoever needs them: few enough for
// a lane each.  What is read is bound by the rows on the path, which are known one after the other:
//   few rows in all: one launch takes all of them, a second one walks down the path;
//   many: a launch for each depth; its workgroups first settle, each for itself and all alike, where the depth before has led.
#include <type_traits>

#include "device_utils.h"
#include "row_penalty.h"
#include "rows_internal.h"
#include "spec_internal.h"

namespace specdraft {

constexpr int kSampleThreads = 256;
constexpr int kMaxParts = 64;

// 2^y for y <= 0: 2^rint(y) times the exponential series of the rest's logarithm, at most ln(2) / 2, to the eleventh power: off by
// 0.3466^12 / 12! = 6e-15 at most
__device__ __forceinline__ double exp2_series(double y) {
  y = fmax(y, -1100.0);
  const double k = __builtin_rint(y), r = y - k;
  constexpr double l = 0.693147180559945309417;
  constexpr double c2 = l * l / 2, c3 = c2 * l / 3, c4 = c3 * l / 4, c5 = c4 * l / 5, c6 = c5 * l / 6, c7 = c6 * l / 7, c8 = c7 * l / 8,
                   c9 = c8 * l / 9, c10 = c9 * l / 10, c11 = c10 * l / 11;
  double p = __builtin_fma(c11, r, c10);
  p = __builtin_fma(p, r, c9);
  p = __builtin_fma(p, r, c8);
  p = __builtin_fma(p, r, c7);
  p = __builtin_fma(p, r, c6);
  p = __builtin_fma(p, r, c5);
  p = __builtin_fma(p, r, c4);
  p = __builtin_fma(p, r, c3);
  p = __builtin_fma(p, r, c2);
  p = __builtin_fma(p, r, l);
  p = __builtin_fma(p, r, 1.0);
  return __builtin_ldexp(p, (int)k);
}

// How a sequence's logits become weights.
struct Heat {
  double per;     // log2(e) / temperature
  bool greedy;    // no temperature: the first maximum has all of the mass
  // of a logit v relative to the largest one `top` (above -inf); v may be -inf
  __device__ __forceinline__ double weight(float v, float top) const {
    if (!(v > SPEC_NEG_INF)) return 0.0;
    if (v == top) return 1.0;   // (also where both are infinite)
    return top == -SPEC_NEG_INF ? 0.0 : exp2_series(((double)v - (double)top) * per);
  }
};
__device__ __forceinline__ Heat heat_of(const float* temperature, int q) {
  const float t = temperature ? temperature[q] : 1.0f;
  return {1.4426950408889634074 / (double)t, !(t > 0.0f)};
}

__device__ __forceinline__ double wave_sum64(double x) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
  return x;
}

// The eight tokens from i on of a row (i a multiple of 8), processed; -inf behind the vocabulary's end and for what is not a number.
// `path`: tokens on the row's path, n_path of them.
template <bool BF16>
__device__ __forceinline__ void processed8(const void* row, int i, int V, const RowPenalty& pen, const int32_t* path, int n_path, float (&v)[8]) {
  typedef uint32_t words __attribute__((ext_vector_type(BF16 ? 4 : 8)));
  typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
  typedef float f32x8 __attribute__((ext_vector_type(8)));
  typedef typename std::conditional<BF16, uint16_t, float>::type T;
  const T* at = static_cast<const T*>(row) + i;
  const bool whole = i + 8 <= V;
  const uint32_t seen = pen.seen ? reinterpret_cast<const uint8_t*>(pen.seen)[i >> 3] : 0u;
  const uint32_t allowed = pen.allowed ? reinterpret_cast<const uint8_t*>(pen.allowed)[i >> 3] : 0xffu;
  if (whole) {
    const words x = load_words<words>(at);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (BF16) v[j] = bf16_bits_to_f32((uint16_t)(x[j / 2] >> (j & 1) * 16));
      else v[j] = __uint_as_float(x[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = i + j < V ? to_f32(at[j]) : SPEC_NEG_INF;
  }
  float bias[8] = {};
  if (pen.bias) {
    if (whole) {
      const f32x8 b = load_words<f32x8>(pen.bias + i);
#pragma unroll
      for (int j = 0; j < 8; ++j) bias[j] = b[j];
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) bias[j] = i + j < V ? pen.bias[i + j] : 0.0f;
    }
  }
  uint32_t touched = pen.counts && !pen.seen ? 0xffu : seen;
  for (int k = 0; k < n_path; ++k) touched |= path[k] >> 3 == i >> 3 ? 1u : 0u;
  int c[8] = {};
  if (touched) {
    if (pen.counts) {
      if (whole) {
        const i32x8 n = load_words<i32x8>(pen.counts + i);
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = !pen.seen || ((seen >> j) & 1) ? n[j] : 0;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = i + j < V && (!pen.seen || ((seen >> j) & 1)) ? pen.counts[i + j] : 0;
      }
    }
    for (int k = 0; k < n_path; ++k) {
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] += path[k] == i + j;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = penalized(v[j], c[j], (seen >> j) & 1, bias[j], (allowed >> j) & 1, pen);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (pen.bias) v[j] = v[j] + bias[j];
      if (!((allowed >> j) & 1)) v[j] = SPEC_NEG_INF;
    }
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = i + j < V && v[j] == v[j] ? v[j] : SPEC_NEG_INF;
}

// Partial of the tokens [begin, end) of a row, by the whole workgroup.
template <bool BF16>
__device__ __forceinline__ void take_part(const SampleJob& p, const void* row, int begin, int end, const RowPenalty& pen, const Heat& heat,
                                          const int32_t* path, int n_path, SamplePart* to) {
  __shared__ float sv[16];
  __shared__ int32_t si[16];
  __shared__ double ss[kSampleThreads / 64];
  const int tid = threadIdx.x;
  float top = SPEC_NEG_INF;
  int32_t first = kIdxNone;
  double sum = 0;
  for (int i = begin + tid * 8; i < end; i += kSampleThreads * 8) {
    float v[8];
    processed8<BF16>(row, i, p.V, pen, path, n_path, v);
    float m = v[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) m = fmaxf(m, v[j]);
    if (m > top) {
      if (top > SPEC_NEG_INF && !heat.greedy) sum *= heat.weight(top, m);
      top = m;
#pragma unroll
      for (int j = 7; j >= 0; --j)
        if (v[j] == m) first = i + j;
    }
    if (!heat.greedy && top > SPEC_NEG_INF) {
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += heat.weight(v[j], top);
    }
  }
  float best = top;
  block_best<kSampleThreads>(best, first, sv, si);
  if (!heat.greedy) {
    sum = top > SPEC_NEG_INF ? sum * heat.weight(top, best) : 0.0;
    sum = wave_sum64(sum);
    if ((tid & 63) == 0) ss[tid >> 6] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < kSampleThreads / 64; ++w) sum += ss[w];
  }
  if (tid == 0) *to = {best, first == kIdxNone ? 0 : first, sum};
}

// A node's token, processed in its parent's row, for every node of a sequence.
template <bool BF16>
__device__ __forceinline__ void take_nodes(const SampleJob& p, int q, int nodes, int32_t* s_node) {
  const int32_t *parent = p.node_parent + (int64_t)q * p.M, *tok = p.node_tok + (int64_t)q * p.M;
  for (int i = threadIdx.x; i < nodes; i += kSampleThreads) {
    s_node[i] = parent[i];
    s_node[p.M + i] = tok[i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nodes; i += kSampleThreads) {
    const int t = s_node[p.M + i], up = s_node[i], row = up >= 0 && up < i ? up + 1 : 0;
    float v = SPEC_NEG_INF;
    if ((uint32_t)t < (uint32_t)p.V) {
      const int at = q * (p.M + 1) + row;
      const RowPenalty pen = penalty_of(p.pen, q, at, p.V);
      const bool bit = pen.seen && ((pen.seen[t >> 5] >> (t & 31)) & 1), allowed = !pen.allowed || ((pen.allowed[t >> 5] >> (t & 31)) & 1);
      int c = pen.counts && (bit || !pen.seen) ? pen.counts[t] : 0;
      for (int node = row - 1, n = 0; node >= 0 && n < kMaxStages; ++n) {
        c += s_node[p.M + node] == t;
        const int x = s_node[node];
        node = x < node ? x : -1;
      }
      if constexpr (BF16) v = bf16_bits_to_f32(static_cast<const uint16_t*>(p.logits)[(int64_t)at * p.V + t]);
      else v = static_cast<const float*>(p.logits)[(int64_t)at * p.V + t];
      v = penalized(v, c, bit, pen.bias ? pen.bias[t] : 0.0f, allowed, pen);
    }
    p.node_v[(int64_t)q * p.M + i] = v == v ? v : SPEC_NEG_INF;
  }
}

// What is settled of a row by its partials and its nodes.
struct Settled {
  int child;           // node that the path goes down to, -1: it ends
  int token;           // that node's, or the last one where it is already known (else -1)
  float logp;          // its logarithm of probability
  float top;           // of the row
  int first;           // its first token of that logit
  double sum;          // S
  double rest;         // where in the others' mass the last token lies
};

// By the first wave; the others get it through LDS.  s_child, s_child_v: the row's nodes' tokens (each once) and their logits.
__device__ __forceinline__ void settle(const SampleJob& p, int q, int row, int nodes, int level, const SamplePart* parts, const Heat& heat,
                                       int32_t* s_child, float* s_child_v, int& n_child, Settled& s) {
  const int lane = threadIdx.x & 63;
  SamplePart mine = {SPEC_NEG_INF, 0, 0.0};
  if (lane < p.parts) mine = parts[lane];
  float top = mine.top;
  int32_t first = mine.top > SPEC_NEG_INF ? mine.first : kIdxNone;
  wave_best(top, first);
  s.child = -1, s.token = -1, s.logp = 0.0f, s.top = top, s.first = first == kIdxNone ? 0 : first, s.sum = 1.0, s.rest = 0.0;
  n_child = 0;
  const bool none = !(top > SPEC_NEG_INF), single = none || heat.greedy;
  if (!single) s.sum = wave_sum64(mine.top > SPEC_NEG_INF ? mine.sum * heat.weight(mine.top, top) : 0.0);
  if (none) s.logp = SPEC_NEG_INF;
  if (single) s.token = s.first;
  float u = p.uniform[(int64_t)q * (p.n + 1) + level];
  u = u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f;   // (what is not in [0, 1) is taken as the nearest that is)
  const double at = (double)u * s.sum;
  if (level < p.n) {
    const int32_t *parent = p.node_parent + (int64_t)q * p.M, *tok = p.node_tok + (int64_t)q * p.M;
    double before_all = 0;
    for (int i0 = 0; i0 < nodes; i0 += 64) {
      const int i = i0 + lane;
      int t = -1;
      float v = SPEC_NEG_INF;
      if (i < nodes) {
        const int up = parent[i];
        t = tok[i], v = p.node_v[(int64_t)q * p.M + i];
        if ((up >= 0 && up < i ? up + 1 : 0) != row || (uint32_t)t >= (uint32_t)p.V) t = -1;
      }
      // (of siblings with the same token the first one counts)
      uint64_t children = __ballot(t >= 0);
      if (!children) continue;
      bool twice = false;
      for (int k = 0; k < n_child; ++k) twice |= s_child[k] == t;
      for (uint64_t rest = children; rest; rest &= rest - 1) {
        const int j = __builtin_ctzll(rest), its = __builtin_amdgcn_readlane(t, j);
        twice |= j < lane && its == t;
      }
      children = __ballot(t >= 0 && !twice);
      const bool counts = t >= 0 && !twice;
      if (counts) {
        const int to = n_child + __popcll(children & ((1ull << lane) - 1));
        s_child[to] = t, s_child_v[to] = v;
      }
      n_child += __popcll(children);
      uint64_t hit;
      double w = 0;
      if (single) {
        hit = __ballot(counts && t == s.first);
      } else {
        w = counts ? heat.weight(v, top) : 0.0;
        double upto = w;   // of the children so far, this one included
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
          const double y = __shfl_up(upto, d);
          if (lane >= d) upto += y;
        }
        hit = __ballot(w > 0 && at < before_all + upto);
        before_all += __shfl(upto, 63);
      }
      if (hit) {
        const int j = __builtin_ctzll(hit);
        s.child = i0 + j;
        s.token = __shfl(t, j);
        if (!single) s.logp = (float)log(__shfl(w, j) / s.sum);
        return;
      }
    }
    s.rest = at - before_all;
  } else {
    s.rest = at;
  }
}

// The part of the row in which the last token lies, and the others' mass before it; by the first wave.
__device__ __forceinline__ int owner_of(const SampleJob& p, const SamplePart* parts, const Heat& heat, const Settled& s, const int32_t* s_child,
                                        const float* s_child_v, int n_child, double& before_part) {
  const int lane = threadIdx.x & 63;
  double mass = 0;
  if (lane < p.parts && parts[lane].top > SPEC_NEG_INF) {
    mass = parts[lane].sum * heat.weight(parts[lane].top, s.top);
    for (int k = 0; k < n_child; ++k)
      if (s_child[k] / p.span == lane) mass -= heat.weight(s_child_v[k], s.top);
  }
  double upto = mass;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const double y = __shfl_up(upto, d);
    if (lane >= d) upto += y;
  }
  const uint64_t hit = __ballot(mass > 0 && s.rest < upto), some = __ballot(mass > 0);
  const int j = hit ? __builtin_ctzll(hit) : some ? 63 - __builtin_clzll(some) : 0;
  before_part = __shfl(upto - mass, j);
  return j;
}

// The first token of a part, children left out, up to which more than `rest` of the mass lies; by the whole workgroup.
template <bool BF16>
__device__ __forceinline__ void find_token(const SampleJob& p, const void* row, int begin, int end, const RowPenalty& pen, const Heat& heat,
                                           const int32_t* path, int n_path, const int32_t* s_child, int n_child, float top, double rest, int otherwise,
                                           int& token, double& weight) {
  __shared__ double s_wave[kSampleThreads / 64], s_weight;
  __shared__ int s_found, s_last;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) s_found = kIdxNone, s_last = -1;
  __syncthreads();
  double carry = 0;
  for (int i0 = begin; i0 < end; i0 += kSampleThreads * 8) {
    const int i = i0 + tid * 8;
    double w[8] = {}, sum = 0;
    int last = -1;
    if (i < end) {
      float v[8];
      processed8<BF16>(row, i, p.V, pen, path, n_path, v);
      uint32_t gone = 0;
      for (int k = 0; k < n_child; ++k) gone |= s_child[k] >> 3 == i >> 3 ? 1u << (s_child[k] & 7) : 0u;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j] = (gone >> j) & 1 ? 0.0 : heat.weight(v[j], top);
        sum += w[j];
        if (w[j] > 0) last = i + j;
      }
    }
    double upto = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const double y = __shfl_up(upto, d);
      if (lane >= d) upto += y;
    }
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    double at = carry + (upto - sum);
#pragma unroll
    for (int x = 0; x < kSampleThreads / 64; ++x) {
      if (x < wave) at += s_wave[x];
      carry += s_wave[x];
    }
    int mine = -1;
    double its = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      at += w[j];
      if (mine < 0 && w[j] > 0 && at > rest) mine = i + j, its = w[j];
    }
    if (mine >= 0) atomicMin(&s_found, mine);
    else if (last >= 0) atomicMax(&s_last, last);
    __syncthreads();
    const int found = s_found;
    if (found != kIdxNone) {
      if (mine == found) s_weight = its;
      __syncthreads();
      token = found, weight = s_weight;
      return;
    }
  }
  // (roundings only lead here: the last one of the part, or the row's largest)
  token = s_last >= 0 ? s_last : otherwise;
  float v[8];
  processed8<BF16>(row, token & ~7, p.V, pen, path, n_path, v);
  weight = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if ((token & 7) == j) weight = heat.weight(v[j], top);
}

// What is emitted for a sequence; by the first wave.
__device__ __forceinline__ void emit(const SampleJob& p, int q, const SampleSlot& s, int token, float logp) {
  const int i = threadIdx.x;
  if (i == 0) p.accept_len[q] = s.level, p.n_out[q] = s.level + 1;
  if (i > p.n) return;
  const int t = i < s.level ? s.tok[i] : i == s.level ? token : -1;
  const int64_t at = (int64_t)q * (p.n + 1) + i;
  p.out_tokens[at] = t;
  p.path_row[at] = i < s.level ? s.path[i] : i == s.level ? s.row : -1;
  if (p.out_logp) p.out_logp[at] = i < s.level ? s.logp[i] : i == s.level ? logp : 0.0f;
  // (whole numbers: their order does not matter)
  if (t >= 0) {
    if (p.counts) atomicAdd(&p.counts[(int64_t)q * p.V + t], 1);
    if (p.seen) atomicOr(&p.seen[(int64_t)q * ((p.V + 31) / 32) + (t >> 5)], 1u << (t & 31));
  }
}

// A sequence that takes no part.
__device__ __forceinline__ void emit_nothing(const SampleJob& p, int q) {
  const int i = threadIdx.x;
  if (i == 0) p.accept_len[q] = p.n_out[q] = 0;
  if (i > p.n) return;
  const int64_t at = (int64_t)q * (p.n + 1) + i;
  p.out_tokens[at] = p.path_row[at] = -1;
  if (p.out_logp) p.out_logp[at] = 0.0f;
}

template <bool BF16>
__device__ __forceinline__ const void* row_of(const SampleJob& p, int q, int row) {
  return static_cast<const uint8_t*>(p.logits) + ((int64_t)q * (p.M + 1) + row) * p.V * (BF16 ? 2 : 4);
}

// Partials of the rows that are known before anything is settled: all of them, or the first of each sequence; and the nodes' logits, by
// one workgroup of each sequence.
template <bool BF16>
__global__ __launch_bounds__(kSampleThreads) void sample_rows_kernel(SampleJob p) {
  extern __shared__ int32_t s_node[];   // [2][M]
  __shared__ int32_t s_path[kMaxStages];
  __shared__ int s_n;
  const int rows = p.all_rows ? p.M + 1 : 1, per = rows * p.parts + 1;
  const int q = blockIdx.x / per, in = blockIdx.x - q * per, r = in / p.parts, part = in - r * p.parts, tid = threadIdx.x;
  const int nodes = p.n_nodes ? min(max(p.n_nodes[q], -1), p.M) : p.M;
  if (r == rows) {
    if (p.M > 0 && nodes > 0) take_nodes<BF16>(p, q, nodes, s_node);
    if (nodes < 0) emit_nothing(p, q);
    if (tid == 0) p.slot[q].done = nodes < 0, p.slot[q].level = 0, p.slot[q].row = 0;
    return;
  }
  if (r > nodes) return;
  const RowPenalty pen = penalty_of(p.pen, q, q * (p.M + 1) + r, p.V);
  int n_path = 0;
  if (r > 0 && p.paths) {
    for (int i = tid; i < r; i += kSampleThreads) {
      s_node[i] = p.node_parent[(int64_t)q * p.M + i];
      s_node[p.M + i] = p.node_tok[(int64_t)q * p.M + i];
    }
    __syncthreads();
    if (tid == 0) {
      int n = 0;
      for (int node = r - 1; node >= 0 && n < kMaxStages;) {
        s_path[n++] = s_node[p.M + node];
        const int up = s_node[node];
        node = up < node ? up : -1;
      }
      s_n = n;
    }
    __syncthreads();
    n_path = s_n;
  }
  take_part<BF16>(p, row_of<BF16>(p, q, r), part * p.span, min(p.V, (part + 1) * p.span), pen, heat_of(p.temperature, q), s_path, n_path,
                  p.part + ((int64_t)q * rows + r) * p.parts + part);
}

// Settles where a sequence's path leads from the rows whose partials are there: from all of them to its end, or from the last one (step - 1
// of them before) one row further, whose partials are then taken.
template <bool BF16>
__global__ __launch_bounds__(kSampleThreads) void sample_walk_kernel(SampleJob p, int step) {
  extern __shared__ int32_t s_child[];   // [M] tokens, [M] logits
  float* s_child_v = reinterpret_cast<float*>(s_child + p.M);
  __shared__ SampleSlot s;
  __shared__ Settled s_set;
  __shared__ int s_n_child, s_owner;
  __shared__ double s_before;
  const int q = blockIdx.x / p.parts, part = blockIdx.x - q * p.parts, tid = threadIdx.x;
  const int nodes = p.n_nodes ? min(max(p.n_nodes[q], -1), p.M) : p.M;
  const Heat heat = heat_of(p.temperature, q);
  SampleSlot* next = p.slot + (int64_t)step * p.batch + q;
  if (tid < (int)(sizeof(SampleSlot) / 4)) reinterpret_cast<int32_t*>(&s)[tid] = reinterpret_cast<const int32_t*>(next - p.batch)[tid];
  __syncthreads();
  if (s.done) {
    if (part == 0 && tid == 0) next->done = 1;
    return;
  }
  for (;;) {
    const SamplePart* parts = p.part + (p.all_rows ? (int64_t)q * (p.M + 1) + s.row : (int64_t)((step - 1) & 1) * p.batch + q) * p.parts;
    if (tid < 64) {
      Settled x;
      int n_child;
      settle(p, q, s.row, nodes, s.level, parts, heat, s_child, s_child_v, n_child, x);
      if (x.child < 0 && x.token < 0) {
        double before_part;
        const int owner = owner_of(p, parts, heat, x, s_child, s_child_v, n_child, before_part);
        if (tid == 0) s_owner = owner, s_before = before_part;
      } else if (tid == 0) {
        s_owner = 0;
      }
      if (tid == 0) s_set = x, s_n_child = n_child;
    }
    __syncthreads();
    if (s_set.child < 0) break;
    if (tid == 0) {
      s.tok[s.level] = s_set.token, s.logp[s.level] = s_set.logp, s.path[s.level] = s.row;
      ++s.level;
      s.row = s_set.child + 1;
    }
    __syncthreads();
    if (p.all_rows) continue;
    if (part == 0 && tid < (int)(sizeof(SampleSlot) / 4)) reinterpret_cast<int32_t*>(next)[tid] = reinterpret_cast<const int32_t*>(&s)[tid];
    const RowPenalty pen = penalty_of(p.pen, q, q * (p.M + 1) + s.row, p.V);
    take_part<BF16>(p, row_of<BF16>(p, q, s.row), part * p.span, min(p.V, (part + 1) * p.span), pen, heat, s.tok, p.paths ? s.level : 0,
                    p.part + ((int64_t)(step & 1) * p.batch + q) * p.parts + part);
    return;
  }
  if (part == 0 && tid == 0 && !p.all_rows) next->done = 1;
  if (s_owner != part) return;
  int token = s_set.token;
  float logp = s_set.logp;
  if (token < 0) {
    const RowPenalty pen = penalty_of(p.pen, q, q * (p.M + 1) + s.row, p.V);
    double weight;
    find_token<BF16>(p, row_of<BF16>(p, q, s.row), part * p.span, min(p.V, (part + 1) * p.span), pen, heat, s.tok, p.paths ? s.level : 0, s_child,
                     s_n_child, s_set.top, s_set.rest - s_before, s_set.first, token, weight);
    logp = (float)log(weight / s_set.sum);
    __syncthreads();   // (counts are read above and written below)
  }
  if (tid < 64) emit(p, q, s, token, logp);
}

// Logits of so many bytes are read whole rather than row by row down the paths.
constexpr int64_t kAllRowsBytes = 32 << 20;

struct SamplePlan {
  int parts, span;
  bool all_rows;
  int64_t part_bytes, node_bytes, slot_bytes;
};
static SamplePlan plan_sample(int batch, int M, int V, bool bf16) {
  SamplePlan a;
  a.span = (int)max((int64_t)4096, (((int64_t)V + kMaxParts - 1) / kMaxParts + 31) & ~(int64_t)31);
  a.parts = (V + a.span - 1) / a.span;
  const int64_t rows = (int64_t)batch * (M + 1);
  a.all_rows = M == 0 || rows * V * (bf16 ? 2 : 4) <= kAllRowsBytes;
  auto padded = [](int64_t x) { return (x + 255) & ~(int64_t)255; };
  a.part_bytes = padded((a.all_rows ? rows : 2 * (int64_t)batch) * a.parts * sizeof(SamplePart));
  a.node_bytes = padded((int64_t)batch * M * sizeof(float));
  a.slot_bytes = padded((int64_t)batch * (kMaxStages + 2) * sizeof(SampleSlot));
  return a;
}

int64_t sample_workspace(int batch, int M, int V, bool bf16) {
  const SamplePlan a = plan_sample(batch, M, V, bf16);
  return a.part_bytes + a.node_bytes + a.slot_bytes;
}

hipError_t launch_sample(SampleJob job, void* workspace, bool bf16, hipStream_t st) {
  const SamplePlan a = plan_sample(job.batch, job.M, job.V, bf16);
  job.parts = a.parts, job.span = a.span, job.all_rows = a.all_rows;
  uint8_t* at = static_cast<uint8_t*>(workspace);
  job.part = reinterpret_cast<SamplePart*>(at);
  job.node_v = reinterpret_cast<float*>(at + a.part_bytes);
  job.slot = reinterpret_cast<SampleSlot*>(at + a.part_bytes + a.node_bytes);
  const size_t smem = (size_t)job.M * 8;
  const unsigned first = (unsigned)job.batch * (unsigned)((a.all_rows ? job.M + 1 : 1) * a.parts + 1), walk = (unsigned)job.batch * (unsigned)a.parts;
  if (bf16) hipLaunchKernelGGL((sample_rows_kernel<true>), dim3(first), dim3(kSampleThreads), smem, st, job);
  else hipLaunchKernelGGL((sample_rows_kernel<false>), dim3(first), dim3(kSampleThreads), smem, st, job);
  hipError_t e = hipGetLastError();
  for (int step = 1; e == hipSuccess && step <= (a.all_rows ? 1 : job.n + 1); ++step) {
    if (bf16) hipLaunchKernelGGL((sample_walk_kernel<true>), dim3(walk), dim3(kSampleThreads), smem, st, job, step);
    else hipLaunchKernelGGL((sample_walk_kernel<false>), dim3(walk), dim3(kSampleThreads), smem, st, job, step);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace specdraft
