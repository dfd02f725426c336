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
constexpr int kPartsAhead = 512;   // partials that are requested before it is known which row's are needed

// How a sequence's logits become weights.
struct Heat {
  double per;     // log2(e) / temperature, 1e-30 at least
  bool greedy;    // no temperature: the first maximum has all of the mass
  // of a finite logit v, or -inf, relative to the largest one `top`, which is finite: 2^y = 2^k 2^r with k the nearest whole number to y (the
  // low bits of y + 1.5 * 2^52) and the exponential series of r's logarithm to the tenth power: off by (ln(2) / 2)^11 / 11! = 2e-13
  // at most.  No branch, so that the series of a thread's tokens run side by side.  What is further below, and -inf, gets 2^-1000.
  __device__ __forceinline__ double weight(float v, float top) const {
    constexpr double l = 0.693147180559945309417, kNear = 6755399441055744.0;
    constexpr double c2 = l * l / 2, c3 = c2 * l / 3, c4 = c3 * l / 4, c5 = c4 * l / 5, c6 = c5 * l / 6, c7 = c6 * l / 7, c8 = c7 * l / 8,
                     c9 = c8 * l / 9, c10 = c9 * l / 10;
    const double y = fmax(((double)v - (double)top) * per, -1000.0), near = y + kNear, r = y - (near - kNear);
    double p = __builtin_fma(c10, r, c9);
    p = __builtin_fma(p, r, c8);
    p = __builtin_fma(p, r, c7);
    p = __builtin_fma(p, r, c6);
    p = __builtin_fma(p, r, c5);
    p = __builtin_fma(p, r, c4);
    p = __builtin_fma(p, r, c3);
    p = __builtin_fma(p, r, c2);
    p = __builtin_fma(p, r, l);
    p = __builtin_fma(p, r, 1.0);
    const uint64_t bits = __builtin_bit_cast(uint64_t, p);
    const uint32_t high = (uint32_t)(bits >> 32) + ((uint32_t)__builtin_bit_cast(uint64_t, near) << 20);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | (uint32_t)bits);
  }
};
__device__ __forceinline__ Heat heat_of(const float* temperature, int q) {
  const float t = temperature ? temperature[q] : 1.0f;
  return {fmax(1.4426950408889634074 / (double)t, 1e-30), !(t > 0.0f)};
}

__device__ __forceinline__ int uniform_of(int x) { return __builtin_amdgcn_readfirstlane(x); }

// a 64-bit number moved by DPP; lanes that get none, and those of rows outside ROWS, get zero
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double dpp_d(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double lane_d(double x, int l) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), l) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, l));
}
// sum of the lanes up to this one
__device__ __forceinline__ double wave_upto(double x) {
  x += dpp_d<0x111>(x);
  x += dpp_d<0x112>(x);
  x += dpp_d<0x114>(x);
  x += dpp_d<0x118>(x);
  x += dpp_d<kDppRowBcast15, 0xa>(x);
  x += dpp_d<kDppRowBcast31, 0xc>(x);
  return x;
}
__device__ __forceinline__ double wave_sum64(double x) { return lane_d(wave_upto(x), 63); }

template <bool BF16>
__device__ __forceinline__ const void* row_of(const SampleJob& p, int q, int row) {
  return static_cast<const uint8_t*>(p.logits) + ((int64_t)q * (p.M + 1) + row) * p.V * (BF16 ? 2 : 4);
}

// The tokens on a row's path, as far as they count.
struct Path {
  const int32_t* tok;   // in LDS
  int n;
};

// Token t of a row, processed: -inf for what is not a number, the largest finite number for +inf.
template <bool BF16>
__device__ __forceinline__ float one_token(const void* row, int t, const RowPenalty& pen, const Path& path) {
  const bool bit = pen.seen && ((pen.seen[t >> 5] >> (t & 31)) & 1), allowed = !pen.allowed || ((pen.allowed[t >> 5] >> (t & 31)) & 1);
  float v;
  if constexpr (BF16) v = bf16_bits_to_f32(static_cast<const uint16_t*>(row)[t]);
  else v = static_cast<const float*>(row)[t];
  int c = pen.counts ? pen.counts[t] : 0;   // (requested with its bit)
  c = bit || !pen.seen ? c : 0;
#pragma unroll 1
  for (int k = 0; k < path.n; ++k) c += path.tok[k] == t;
  v = penalized(v, c, bit, pen.bias ? pen.bias[t] : 0.0f, allowed, pen);
  return v == v ? fminf(v, __FLT_MAX__) : SPEC_NEG_INF;
}

// A thread's 16 tokens of a row from `first` on, a multiple of 16: what is requested before they are worked on.
template <bool BF16>
struct Sixteen {
  typedef uint32_t words __attribute__((ext_vector_type(8)));
  typedef float f32x8 __attribute__((ext_vector_type(8)));
  typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
  uint32_t seen, allowed;        // bits
  words x[BF16 ? 1 : 2];
  f32x8 bias[2];
  i32x8 c[2];                    // where one of eight was seen
  static __device__ __forceinline__ uint32_t bits(const uint32_t* of, int first, int V) { return (of[min(first, V - 1) >> 5] >> (first & 16)) & 0xffffu; }
  __device__ __forceinline__ void load_seen(const RowPenalty& pen, int first, int V) { seen = pen.seen ? bits(pen.seen, first, V) : 0u; }
  __device__ __forceinline__ void load(const void* row, const RowPenalty& pen, int first, int V) {
    allowed = pen.allowed ? bits(pen.allowed, first, V) : ~0u;
    if (first + 16 <= V) {
      const uint8_t* at = static_cast<const uint8_t*>(row) + (int64_t)first * (BF16 ? 2 : 4);
#pragma unroll
      for (int j = 0; j < (BF16 ? 1 : 2); ++j) x[j] = load_words<words>(at + j * 32);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        c[u] = (i32x8){0, 0, 0, 0, 0, 0, 0, 0};
        if (pen.counts && (!pen.seen || (seen >> 8 * u) & 0xff)) c[u] = load_words<i32x8>(pen.counts + first + 8 * u);
      }
      if (pen.bias) bias[0] = load_words<f32x8>(pen.bias + first), bias[1] = load_words<f32x8>(pen.bias + first + 8);
    } else if (first < V) {   // (one thread of a row at most)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const int i = first + j;
        if constexpr (BF16) {
          const uint32_t e = i < V ? static_cast<const uint16_t*>(row)[i] : 0u;
          x[0][j / 2] = j & 1 ? x[0][j / 2] | e << 16 : e;
        } else {
          x[j / 8][j % 8] = i < V ? static_cast<const uint32_t*>(row)[i] : 0u;
        }
        if (pen.bias) bias[j / 8][j % 8] = i < V ? pen.bias[i] : 0.0f;
        c[j / 8][j % 8] = i < V && pen.counts ? pen.counts[i] : 0;
      }
    }
  }
  __device__ __forceinline__ float raw(int j) const {
    if constexpr (BF16) return bf16_bits_to_f32((uint16_t)(x[0][j / 2] >> (j & 1) * 16));
    else return __uint_as_float(x[j / 8][j % 8]);
  }
};

// Largest logit, its first token (where all of the mass is one token's) and sum relative to it of this thread's tokens, those of the list
// s_child left out.  x holds the first 16.
template <bool BF16>
__device__ __forceinline__ SamplePart take_run(const void* row, int begin, int run, int V, const RowPenalty& pen, const Heat& heat, const Path& path,
                                               Sixteen<BF16>& x, const int32_t* s_child, int n_child) {
  SamplePart of = {SPEC_NEG_INF, kIdxNone, 0.0};
#pragma unroll 1
  for (int k = 0; k < run; k += 16) {
    const int first = begin + k;
    if (k > 0) x.load_seen(pen, first, V), x.load(row, pen, first, V);
    uint32_t here = first < V ? 0xffffu >> max(first + 16 - V, 0) : 0u, on_path = 0;
#pragma unroll 1
    for (int c = 0; c < path.n; ++c) on_path |= (uint32_t)(path.tok[c] - first) < 16u ? 1u << (path.tok[c] - first) : 0u;
#pragma unroll 1
    for (int c = 0; c < n_child; ++c) here &= ~((uint32_t)(s_child[c] - first) < 16u ? 1u << (s_child[c] - first) : 0u);
    here &= x.allowed;
    float v[16], m = SPEC_NEG_INF;
#pragma unroll
    for (int j = 0; j < 16; ++j) v[j] = x.raw(j);
    if (((x.seen & 0xffffu) | on_path) || (pen.counts && !pen.seen)) {
      if (on_path) {   // (few lanes)
#pragma unroll 1
        for (int c = 0; c < path.n; ++c) {
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            // (what was emitted before counts where its bit is set, bit j; a token that the path has had has bit 16 + j, and its count goes on)
            if (path.tok[c] - first == j) x.c[j / 8][j % 8] = (pen.seen && !((x.seen >> j) & 0x10001u) ? 0 : x.c[j / 8][j % 8]) + 1, x.seen |= 0x10000u << j;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const bool bit = (x.seen >> j) & 1;
        const int c = !pen.seen || bit || ((x.seen >> (16 + j)) & 1) ? x.c[j / 8][j % 8] : 0;
        v[j] = penalized(v[j], c, bit, pen.bias ? x.bias[j / 8][j % 8] : 0.0f, true, pen);
      }
    } else if (pen.bias) {
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = v[j] + x.bias[j / 8][j % 8];
    }
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      // (not a number: the smaller operand; +inf: the largest finite number)
      v[j] = (here >> j) & 1 ? fminf(fmaxf(v[j], SPEC_NEG_INF), __FLT_MAX__) : SPEC_NEG_INF;
      m = fmaxf(m, v[j]);
    }
    if (heat.greedy) {
      if (m > of.top) {
        of.top = m;
#pragma unroll
        for (int j = 15; j >= 0; --j) of.first = v[j] == m ? first + j : of.first;
      }
      continue;
    }
    if (m > of.top) of.sum = of.top > SPEC_NEG_INF ? of.sum * heat.weight(of.top, m) : 0.0, of.top = m;
    if (of.top > SPEC_NEG_INF) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        double w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = heat.weight(v[u * 8 + j], of.top);
        of.sum += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
      }
    }
  }
  return of;
}

// Partial of a part from its threads', by the whole workgroup.
__device__ __forceinline__ void join_runs(const Heat& heat, SamplePart of, SamplePart* to) {
  __shared__ float sv[16];
  __shared__ int32_t si[16];
  __shared__ double ss[kSampleThreads / 64];
  const int tid = threadIdx.x;
  float best = of.top;
  block_best<kSampleThreads>(best, of.first, sv, si);
  double sum = 0;
  if (!heat.greedy) {
    sum = wave_sum64(of.top > SPEC_NEG_INF ? of.sum * heat.weight(of.top, best) : 0.0);
    if ((tid & 63) == 0) ss[tid >> 6] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < kSampleThreads / 64; ++w) sum += ss[w];
  }
  if (tid == 0) *to = {best, of.first == kIdxNone ? 0 : of.first, sum};
}

// A node's token, processed in its parent's row, for every node of a sequence.
template <bool BF16>
__device__ __forceinline__ void take_nodes(const SampleJob& p, int q, int nodes, int32_t* s_node) {
  __shared__ int32_t s_up[kSampleThreads][kMaxStages];
  const int32_t *parent = p.node_parent + (int64_t)q * p.M, *tok = p.node_tok + (int64_t)q * p.M;
  const int tid = threadIdx.x;
  for (int i = tid; i < nodes; i += kSampleThreads) {
    s_node[i] = parent[i];
    s_node[p.M + i] = tok[i];
  }
  __syncthreads();
  for (int i = tid; i < nodes; i += kSampleThreads) {
    const int t = s_node[p.M + i], up = s_node[i], row = up >= 0 && up < i ? up + 1 : 0;
    float v = SPEC_NEG_INF;
    if ((uint32_t)t < (uint32_t)p.V) {
      Path path = {s_up[tid], 0};
      if (p.paths) {
#pragma unroll 1
        for (int node = row - 1; node >= 0 && path.n < kMaxStages; ++path.n) {
          s_up[tid][path.n] = s_node[p.M + node];
          const int x = s_node[node];
          node = x < node ? x : -1;
        }
      }
      v = one_token<BF16>(row_of<BF16>(p, q, row), t, penalty_of(p.pen, q, q * (p.M + 1) + row, p.V), path);
    }
    p.node_v[(int64_t)q * p.M + i] = v;
  }
}

// What is settled of a row by its partials and its nodes.
struct Settled {
  int child;           // node that the path goes down to, -1: it ends
  int token;           // that node's, or the last one where it is already known (else -1)
  double weight;       // its w
  float top;           // of the row
  int first;           // its first token of that logit
  double sum;          // S
  double rest;         // where in the others' mass the last token lies
};

// A lane's node of 64.
struct LaneNode {
  int row, token;      // its parent's row; -1: no node, or a token that is none
  float v;
  __device__ __forceinline__ void load(const SampleJob& p, int q, int nodes, int i) {
    row = -1, token = -1, v = SPEC_NEG_INF;
    if (i < nodes) {
      const int64_t at = (int64_t)q * p.M + i;
      const int up = p.node_parent[at], t = p.node_tok[at];
      v = p.node_v[at];
      if ((uint32_t)t < (uint32_t)p.V) row = up >= 0 && up < i ? up + 1 : 0, token = t;
    }
  }
};

// By the first wave; the others get it through LDS.  mine: the lane's partial of the row; node0: its node of the first 64.  s_child, s_child_w:
// the row's nodes' tokens (each once) and their weights.
__device__ __forceinline__ void settle(const SampleJob& p, int q, int row, int nodes, int level, float u, const SamplePart& mine, const LaneNode& node0,
                                       const Heat& heat, int32_t* s_child, double* s_child_w, int& n_child, Settled& s) {
  const int lane = threadIdx.x & 63;
  float top = mine.top;
  int32_t first = mine.top > SPEC_NEG_INF ? mine.first : kIdxNone;
  wave_best(top, first);
  s.child = -1, s.token = -1, s.weight = 1.0, s.top = top, s.first = first == kIdxNone ? 0 : first, s.sum = 1.0, s.rest = 0.0;
  n_child = 0;
  const bool none = !(top > SPEC_NEG_INF), single = none || heat.greedy;
  if (!single) s.sum = wave_sum64(mine.top > SPEC_NEG_INF ? mine.sum * heat.weight(mine.top, top) : 0.0);
  if (none) s.weight = 0.0;
  if (single) s.token = s.first;
  u = u > 0.0f ? fminf(u, 0x1.fffffep-1f) : 0.0f;   // (what is not in [0, 1) is taken as the nearest that is)
  const double at = (double)u * s.sum;
  double before_all = 0;
  for (int i0 = 0; level < p.n && i0 < nodes; i0 += 64) {
    LaneNode x = node0;
    if (i0 > 0) x.load(p, q, nodes, i0 + lane);
    // (of siblings with the same token the first one counts)
    uint64_t children = __ballot(x.row == row);
    if (!children) continue;
    bool twice = false;
    for (int k = 0; k < n_child; ++k) twice |= s_child[k] == x.token;
    for (uint64_t rest = children; rest; rest &= rest - 1) {
      const int j = __builtin_ctzll(rest), its = __builtin_amdgcn_readlane(x.token, j);
      twice |= j < lane && its == x.token;
    }
    const bool counts = x.row == row && !twice;
    children = __ballot(counts);
    uint64_t hit;
    double w = 0;
    if (single) {
      hit = __ballot(counts && x.token == s.first);
    } else {
      w = heat.weight(x.v, top);
      w = counts && x.v > SPEC_NEG_INF ? w : 0.0;
      const double upto = wave_upto(w);   // of the children so far, this one included
      hit = __ballot(w > 0 && at < before_all + upto);
      before_all += lane_d(upto, 63);
    }
    if (counts) {
      const int to = n_child + __popcll(children & ((1ull << lane) - 1));
      s_child[to] = x.token, s_child_w[to] = w;
    }
    n_child += __popcll(children);
    if (hit) {
      const int j = __builtin_ctzll(hit);
      s.child = i0 + j;
      s.token = __builtin_amdgcn_readlane(x.token, j);
      if (!single) s.weight = lane_d(w, j);
      return;
    }
  }
  s.rest = at - before_all;
}

// The part of the row in which the last token lies, and the others' mass before it; by the first wave.
__device__ __forceinline__ int owner_of(const SampleJob& p, const SamplePart& mine, const Heat& heat, const Settled& s, const int32_t* s_child,
                                        const double* s_child_w, int n_child, double& before_part) {
  const int lane = threadIdx.x & 63;
  double mass = mine.top > SPEC_NEG_INF ? mine.sum * heat.weight(mine.top, s.top) : 0.0;
  for (int k = 0; k < n_child; ++k)
    mass -= (uint32_t)(s_child[k] - lane * p.span) < (uint32_t)p.span ? s_child_w[k] : 0.0;
  const double upto = wave_upto(mass);
  const uint64_t hit = __ballot(mass > 0 && s.rest < upto), some = __ballot(mass > 0);
  const int j = hit ? __builtin_ctzll(hit) : some ? 63 - __builtin_clzll(some) : 0;
  before_part = lane_d(upto - mass, j);
  return j;
}

// The first token of a part, children left out, up to which more than `rest` of the mass lies; by the whole workgroup, whose threads hold
// the partials `of` of their runs.
template <bool BF16>
__device__ __forceinline__ void find_token(const void* row, int begin, int run, int V, const RowPenalty& pen, const Heat& heat, const Path& path, const SamplePart& of,
                                           const int32_t* s_child, const double* s_child_w, int n_child, float top, double rest, int& token,
                                           double& weight) {
  __shared__ double s_wave[kSampleThreads / 64], s_before;
  __shared__ int s_at, s_last;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const double sum = of.top > SPEC_NEG_INF ? of.sum * heat.weight(of.top, top) : 0.0;
  const double upto = wave_upto(sum);
  if (lane == 63) s_wave[wave] = upto;
  if (tid == 0) s_at = kIdxNone, s_last = -1;
  __syncthreads();
  double at = upto - sum;
#pragma unroll
  for (int w = 0; w < kSampleThreads / 64; ++w)
    if (w < wave) at += s_wave[w];
  // the first thread up to which there is more, if roundings leave none the last one that has any
  if (of.top > SPEC_NEG_INF) {
    if (at + sum > rest) atomicMin(&s_at, tid);
    atomicMax(&s_last, tid);
  }
  __syncthreads();
  const int who = s_at != kIdxNone ? s_at : s_last;
  if (tid == who) s_before = at;
  __syncthreads();
  if (tid >= 64) return;
  if (who < 0) {   // (roundings only lead here: the children have all of the mass)
    token = 0, weight = 0;
    for (int k = 0; k < n_child; ++k)
      if (s_child_w[k] > 0) token = s_child[k], weight = s_child_w[k];
    return;
  }
  // its tokens, one to a lane; the first one up to which there is more, else the last one
  double before_all = s_before;
  for (int k = 0; k < run; k += 64) {
    const int t = begin + who * run + k + lane;
    double w = 0;
    if (k + lane < run && t < V) {
      bool out = false;
#pragma unroll 1
      for (int c = 0; c < n_child; ++c) out |= s_child[c] == t;
      const float v = one_token<BF16>(row, t, pen, path);
      if (!out && v > SPEC_NEG_INF) w = heat.weight(v, top);
    }
    const double sum_to = wave_upto(w);
    const uint64_t some = __ballot(w > 0), hit = __ballot(w > 0 && before_all + sum_to > rest);
    if (some) {
      const int j = hit ? __builtin_ctzll(hit) : 63 - __builtin_clzll(some);
      token = begin + who * run + k + j;
      weight = lane_d(w, j);
    }
    if (hit) return;
    before_all += lane_d(sum_to, 63);
  }
}

// What is emitted for a sequence; by the first wave.
__device__ __forceinline__ void emit(const SampleJob& p, int q, const SampleSlot& s, int token, double weight, double sum) {
  const int i = threadIdx.x;
  if (i == 0) p.accept_len[q] = s.level, p.n_out[q] = s.level + 1;
  if (i > p.n) return;
  const int t = i < s.level ? s.tok[i] : i == s.level ? token : -1;
  const int64_t at = (int64_t)q * (p.n + 1) + i;
  p.out_tokens[at] = t;
  p.path_row[at] = i < s.level ? s.path[i] : i == s.level ? s.row : -1;
  if (p.out_logp) p.out_logp[at] = i <= s.level ? (float)log(i < s.level ? s.weight[i] / s.sum[i] : weight / sum) : 0.0f;
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

// Partials of the rows that are known before anything is settled: all of them, or the first of each sequence; and the nodes' logits, by
// one workgroup of each sequence.
template <bool BF16>
__global__ __launch_bounds__(kSampleThreads, 4) void sample_rows_kernel(SampleJob p) {
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
  const void* row = row_of<BF16>(p, q, r);
  const int begin = part * p.span + tid * p.run;
  Sixteen<BF16> x;
  x.load_seen(pen, begin, p.V);
  x.load(row, pen, begin, p.V);
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
  }
  const Heat heat = heat_of(p.temperature, q);
  const SamplePart of = take_run<BF16>(row, begin, p.run, p.V, pen, heat, {s_path, r > 0 && p.paths ? s_n : 0}, x, nullptr, 0);
  join_runs(heat, of, p.part + ((int64_t)q * rows + r) * p.parts + part);
}

// Settles where a sequence's path leads from the rows whose partials are there: from all of them to its end, or from the last one (step - 1
// of them before) one row further, whose partials are then taken.
template <bool BF16>
__global__ __launch_bounds__(kSampleThreads, 3) void sample_walk_kernel(SampleJob p, int step) {
  extern __shared__ double s_child_w[];   // [M] weights, [M] tokens
  int32_t* s_child = reinterpret_cast<int32_t*>(s_child_w + p.M);
  __shared__ SampleSlot s;
  __shared__ Settled s_set;
  __shared__ int s_n_child, s_owner;
  __shared__ double s_before;
  __shared__ SamplePart s_part[kPartsAhead];
  const int q = blockIdx.x / p.parts, part = blockIdx.x - q * p.parts, tid = threadIdx.x;
  const int nodes = p.n_nodes ? min(max(p.n_nodes[q], -1), p.M) : p.M;
  const Heat heat = heat_of(p.temperature, q);
  SampleSlot* next = p.slot + (int64_t)step * p.batch + q;
  constexpr int kWords = sizeof(SampleSlot) / 4;
  // (requested before it is known where the path has led: the row's partials, the nodes, what the sequence says of this thread's tokens)
  const SamplePart* all = p.part + (p.all_rows ? (int64_t)q * (p.M + 1) : (int64_t)((step - 1) & 1) * p.batch + q) * p.parts;
  const int ahead = (p.all_rows ? max(nodes + 1, 0) : 1) * p.parts;
  LaneNode node0;
  if (tid < 64) node0.load(p, q, nodes, tid);
  int32_t word = 0;
  if (tid >= 64 && tid < 64 + kWords) word = reinterpret_cast<const int32_t*>(next - p.batch)[tid - 64];
  for (int i = tid; i < min(ahead, kPartsAhead); i += kSampleThreads) s_part[i] = all[i];
  RowPenalty pen = penalty_of(p.pen, q, q * (p.M + 1), p.V);   // (of row 0: bias and what is the sequence's)
  const int mine = part * p.span + tid * p.run;
  Sixteen<BF16> x;
  x.load_seen(pen, mine, p.V);
  float u = 0;
  if (tid <= p.n) u = p.uniform[(int64_t)q * (p.n + 1) + tid];
  const int32_t mask = p.pen.allowed && (tid & 63) <= p.M ? p.pen.mask_row[(int64_t)q * (p.M + 1) + (tid & 63)] : -1;   // of the first 64 rows
  if (tid >= 64 && tid < 64 + kWords) reinterpret_cast<int32_t*>(&s)[tid - 64] = word;
  __syncthreads();
  if (s.done) {
    if (part == 0 && tid == 0) next->done = 1;
    return;
  }
  for (;;) {
    if (tid < 64) {
      SamplePart of = {SPEC_NEG_INF, 0, 0.0};
      const int at = (p.all_rows ? s.row : 0) * p.parts + tid;
      if (tid < p.parts) of = at < kPartsAhead ? s_part[at] : all[at];
      Settled y;
      int n_child;
      settle(p, q, s.row, nodes, s.level, lane_f(u, uniform_of(s.level)), of, node0, heat, s_child, s_child_w, n_child, y);
      if (y.child < 0 && y.token < 0) {
        double before_part;
        const int owner = owner_of(p, of, heat, y, s_child, s_child_w, n_child, before_part);
        if (tid == 0) s_owner = owner, s_before = before_part;
      } else if (tid == 0) {
        s_owner = 0;
      }
      if (tid == 0) {
        s_set = y, s_n_child = n_child;
        if (y.child >= 0) {
          s.tok[s.level] = y.token, s.weight[s.level] = y.weight, s.sum[s.level] = y.sum, s.path[s.level] = s.row;
          ++s.level;
          s.row = y.child + 1;
        }
      }
    }
    __syncthreads();
    if (s_set.child < 0) break;
    if (!p.all_rows) break;
    __syncthreads();   // (s_set is read above and written below)
  }
  const bool down = s_set.child >= 0;   // only a row further
  if (!down && part == 0 && tid == 0 && !p.all_rows) next->done = 1;
  if (!down && s_owner != part) return;
  int token = s_set.token;
  double weight = s_set.weight;
  if (down || token < 0) {
    const int r = uniform_of(s.row);
    if (p.pen.allowed) {
      const int m = r < 64 ? __builtin_amdgcn_readlane(mask, r) : p.pen.mask_row[(int64_t)q * (p.M + 1) + r];
      pen.allowed = m >= 0 && m < p.pen.n_allowed ? p.pen.allowed + (int64_t)m * ((p.V + 31) / 32) : nullptr;
    }
    const void* row = row_of<BF16>(p, q, r);
    x.load(row, pen, mine, p.V);
    const Path path = {s.tok, p.paths ? s.level : 0};
    const SamplePart of = take_run<BF16>(row, mine, p.run, p.V, pen, heat, path, x, s_child, down ? 0 : s_n_child);
    if (down) {
      if (part == 0 && tid < kWords) reinterpret_cast<int32_t*>(next)[tid] = reinterpret_cast<const int32_t*>(&s)[tid];
      join_runs(heat, of, p.part + ((int64_t)(step & 1) * p.batch + q) * p.parts + part);
      return;
    }
    find_token<BF16>(row, part * p.span, p.run, p.V, pen, heat, path, of, s_child, s_child_w, s_n_child, s_set.top, s_set.rest - s_before, token, weight);
    // (counts have been read by the wave that writes them)
  }
  if (tid < 64) emit(p, q, s, token, weight, s_set.sum);
}

// Up to so many logits are all taken in one launch, more row by row down the paths, a launch for each depth.  All rows / paths, us, where
// half of the drafted tokens or more are kept: trees of 49 rows, vocabulary 32,000, float32, 4, 8, 12, 16 and 32 sequences (6, 13, 19, 25 and 50
// million logits) 35.8 / 55.2, 43.6 / 60.8, 53.0 / 62.4, 63.6 / 63.6 and 100 / 69; of 65 rows, 128,256, bfloat16, 1, 2, 3, 4 and 8 sequences (8, 17, 25, 33
// and 67 million) 36.2 / 52.6, 48.9 / 61.2, 62.4 / 64.5, 73.8 / 66.2 and 121 / 73; of 97 rows, 32,000, bfloat16, 4, 8 and 16 (12, 25 and 50 million) 40.6 / 60.8,
// 55.4 / 60.6 and 85.5 / 65.2.  So they meet between 25 and 30 million in either type, and from here to there the paths cost up to 9 us more; where
// paths end early they are faster, and all rows are not.
constexpr int64_t kAllRowsLogits = 1 << 24;

struct SamplePlan {
  int parts, span, run;   // tokens of a part, and of a thread of it
  bool all_rows;
  int64_t part_bytes, node_bytes, slot_bytes;
};
static SamplePlan plan_sample(int batch, int M, int V) {
  SamplePlan a;
  const int64_t rows = (int64_t)batch * (M + 1);
  a.all_rows = M == 0 || rows * V <= kAllRowsLogits;
  const int64_t least = ((int64_t)V + kMaxParts * kSampleThreads - 1) / (kMaxParts * kSampleThreads);   // tokens of a thread
  a.run = (int)max((int64_t)16, (least + 15) & ~(int64_t)15);
  a.span = a.run * kSampleThreads;
  a.parts = (int)(((int64_t)V + a.span - 1) / a.span);
  auto padded = [](int64_t x) { return (x + 255) & ~(int64_t)255; };
  // no less than fewer sequences or rows need, whose partials may all be held at once: the largest call's buffer serves the others
  const int64_t held = max(max((int64_t)batch, min(rows, kAllRowsLogits / V)), a.all_rows ? (int64_t)0 : 2 * (int64_t)batch);
  a.part_bytes = padded(held * a.parts * sizeof(SamplePart));
  a.node_bytes = padded((int64_t)batch * M * sizeof(float));
  a.slot_bytes = padded((int64_t)batch * (kMaxStages + 2) * sizeof(SampleSlot));
  return a;
}

int64_t sample_workspace(int batch, int M, int V) {
  const SamplePlan a = plan_sample(batch, M, V);
  return a.part_bytes + a.node_bytes + a.slot_bytes;
}

hipError_t launch_sample(SampleJob job, void* workspace, bool bf16, hipStream_t st) {
  const SamplePlan a = plan_sample(job.batch, job.M, job.V);
  job.parts = a.parts, job.span = a.span, job.run = a.run, job.all_rows = a.all_rows;
  uint8_t* at = static_cast<uint8_t*>(workspace);
  job.part = reinterpret_cast<SamplePart*>(at);
  job.node_v = reinterpret_cast<float*>(at + a.part_bytes);
  job.slot = reinterpret_cast<SampleSlot*>(at + a.part_bytes + a.node_bytes);
  const unsigned first = (unsigned)job.batch * (unsigned)((a.all_rows ? job.M + 1 : 1) * a.parts + 1), walk = (unsigned)job.batch * (unsigned)a.parts;
  if (bf16) hipLaunchKernelGGL((sample_rows_kernel<true>), dim3(first), dim3(kSampleThreads), job.M * 8, st, job);
  else hipLaunchKernelGGL((sample_rows_kernel<false>), dim3(first), dim3(kSampleThreads), job.M * 8, st, job);
  hipError_t e = hipGetLastError();
  for (int step = 1; e == hipSuccess && step <= (a.all_rows ? 1 : job.n + 1); ++step) {
    if (bf16) hipLaunchKernelGGL((sample_walk_kernel<true>), dim3(walk), dim3(kSampleThreads), job.M * 12, st, job, step);
    else hipLaunchKernelGGL((sample_walk_kernel<false>), dim3(walk), dim3(kSampleThreads), job.M * 12, st, job, step);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace specdraft
