// The logits of a token tree's rows: penalties, biases and masks, the first maximum of every row, and the path of nodes
// that the base model agrees with.
//   c = counts[t] + occurrences of t on the row's path;  seen = its bit, or c > 0
//   v = logits[t];  seen: v = v > 0 ? v / repetition : v * repetition;  v -= frequency * c;  c > 0: v -= presence;
//   v += bias[t];  not allowed: v = -inf
#include <type_traits>

#include "device_utils.h"
#include "rows_internal.h"
#include "spec_internal.h"

namespace specdraft {

constexpr int kRowThreads = 512;
constexpr int kRowChunks = 4;   // chunks of 8 tokens that a thread has in flight

// eight neighbours; rows of an odd length start anywhere, so their words are not aligned to 16 bytes (the compiler's memcpy is one
// 16-byte load all the same)
template <typename T>
__device__ __forceinline__ T load_words(const void* from) {
  T x;
  __builtin_memcpy(&x, from, sizeof(T));
  return x;
}

// What changes one sequence's logits (row by row: allowed).
struct RowPenalty {
  const int32_t* counts;
  const uint32_t *seen, *allowed;
  const float* bias;
  float rep, pres, freq;
};

// A token that was seen, or is on the path, by the whole formula; c: its occurrences.
__device__ __forceinline__ float penalized(float v, int i, int c, bool bit, const RowPenalty& pen) {
// (a product and a difference are rounded one by one: what is chosen must not hang on the compiler's choice)
#pragma clang fp contract(off)
  if (bit || c > 0) v = v > 0.0f ? v / pen.rep : v * pen.rep;
  v = v - pen.freq * (float)c;
  if (c > 0) v = v - pen.pres;
  if (pen.bias) v = v + pen.bias[i];
  if (pen.allowed && !((pen.allowed[i >> 5] >> (i & 31)) & 1)) v = SPEC_NEG_INF;
  return v;
}

// One workgroup per row.  Few tokens of a row were seen or are on its path: TOUCHED tokens.  The others only take a bias and a
// mask, eight at a time; the touched ones are left out there (their logits stay as they are) and done one by one from the bits.
template <bool BF16, bool OUT>
__global__ __launch_bounds__(kRowThreads, 4) void logits_kernel(LogitsJob p) {
  typedef uint32_t words __attribute__((ext_vector_type(BF16 ? 4 : 8)));
  typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
  typedef float floatx8 __attribute__((ext_vector_type(8)));
  typedef typename std::conditional<BF16, uint16_t, float>::type T;
  extern __shared__ int32_t s_node[];   // parents, tokens [M]
  __shared__ float sv[16];
  __shared__ int32_t si[16];
  __shared__ int32_t s_path[kMaxStages];
  __shared__ int s_n;
  const int R = p.M + 1, q = blockIdx.x / R, r = blockIdx.x - q * R, tid = threadIdx.x, lane = tid & 63, V = p.V;
  const int nodes = p.n_nodes ? min(max(p.n_nodes[q], -1), p.M) : p.M;
  if (r > nodes) {
    if (!OUT && tid == 0) p.greedy[blockIdx.x] = -1;
    return;
  }
  const T* row = static_cast<const T*>(p.logits) + (int64_t)blockIdx.x * V;
  T* out = OUT ? static_cast<T*>(p.out) + (int64_t)blockIdx.x * V : nullptr;
  words x[kRowChunks];
  auto load = [&](int i0) {
#pragma unroll
    for (int u = 0; u < kRowChunks; ++u) {
      const int i = i0 + u * kRowThreads * 8;
      if (i + 8 <= V) {
        x[u] = load_words<words>(row + i);
      } else if (i < V) {   // the row's last tokens
        T e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = i + j < V ? row[i + j] : T(0);
        x[u] = load_words<words>(e);
      }
    }
  };
  load(tid * 8);

  // ---- the tokens on the row's path ----
  int n_path = 0;
  if (p.node_tok && r > 0) {
    for (int i = tid; i < r; i += kRowThreads) {
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
    n_path = __builtin_amdgcn_readfirstlane(s_n);
  }
  int path[kMaxStages];   // in scalar registers; -1: none
#pragma unroll
  for (int j = 0; j < kMaxStages; ++j) path[j] = j < n_path ? __builtin_amdgcn_readfirstlane(s_path[j]) : -1;
  const int n_words = (V + 31) / 32;
  RowPenalty pen;
  pen.counts = p.pen.counts ? p.pen.counts + (int64_t)q * V : nullptr;
  pen.seen = p.pen.seen ? p.pen.seen + (int64_t)q * n_words : nullptr;
  pen.rep = p.pen.repetition ? p.pen.repetition[q] : 1.0f, pen.pres = p.pen.presence ? p.pen.presence[q] : 0.0f;
  pen.freq = p.pen.frequency ? p.pen.frequency[q] : 0.0f;
  const int bias_row = p.pen.bias ? p.pen.bias_row[q] : -1, mask_row = p.pen.allowed ? p.pen.mask_row[blockIdx.x] : -1;
  pen.bias = bias_row >= 0 && bias_row < p.pen.n_bias ? p.pen.bias + (int64_t)bias_row * V : nullptr;
  pen.allowed = mask_row >= 0 && mask_row < p.pen.n_allowed ? p.pen.allowed + (int64_t)mask_row * n_words : nullptr;

  // ---- untouched tokens ----
  float bv = SPEC_NEG_INF;
  int32_t bi = kIdxNone;
  for (int i0 = tid * 8; i0 - tid * 8 < V; i0 += kRowThreads * 8 * kRowChunks) {
    uint32_t touched[kRowChunks], ok[kRowChunks];
#pragma unroll
    for (int u = 0; u < kRowChunks; ++u) {
      const int i = i0 + u * kRowThreads * 8;
      touched[u] = 0, ok[u] = 0xff;
      if (i < V) {
        // (byte i / 8 of a row of words; a last byte may hold bits behind the row, which `left` takes out)
        if (pen.seen) touched[u] = reinterpret_cast<const uint8_t*>(pen.seen)[i >> 3];
        if (pen.allowed) ok[u] = reinterpret_cast<const uint8_t*>(pen.allowed)[i >> 3];
        if (pen.counts && !pen.seen) {
          if (i + 8 <= V) {
            const i32x8 c = load_words<i32x8>(pen.counts + i);
#pragma unroll
            for (int j = 0; j < 8; ++j) touched[u] |= c[j] ? 1u << j : 0u;
          } else {
            for (int j = 0; i + j < V; ++j) touched[u] |= pen.counts[i + j] ? 1u << j : 0u;
          }
        }
      }
#pragma unroll
      for (int j = 0; j < kMaxStages; ++j) {
        // the wave's 512 tokens hold it: one lane's chunk does
        const uint32_t at = (uint32_t)path[j] - (uint32_t)__builtin_amdgcn_readfirstlane(i - lane * 8);
        if (j < n_path && at < 512u) touched[u] |= lane == (int)(at >> 3) ? 1u << (at & 7) : 0u;
      }
    }
#pragma unroll
    for (int u = 0; u < kRowChunks; ++u) {
      const int i = i0 + u * kRowThreads * 8;
      if (i >= V) continue;
      const int left = min(V - i, 8);
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (BF16) v[j] = bf16_bits_to_f32((uint16_t)(x[u][j / 2] >> (j & 1) * 16));
        else v[j] = __uint_as_float(x[u][j]);
      }
      if (pen.bias) {
        floatx8 y = {0, 0, 0, 0, 0, 0, 0, 0};
        if (left == 8) {
          y = load_words<floatx8>(pen.bias + i);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = j < left ? pen.bias[i + j] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += OUT && ((touched[u] >> j) & 1) ? 0.0f : y[j];
      }
      if constexpr (OUT) {
        const uint32_t gone = ~ok[u] & ~touched[u] & 0xff;
        if (gone) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = (gone >> j) & 1 ? SPEC_NEG_INF : v[j];
        }
        if (!pen.bias && !gone && p.out == p.logits) continue;
        words w;
        if constexpr (BF16) {
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = f32_to_bf16_pair(v[2 * j], v[2 * j + 1]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[j]);
        }
        if (left == 8) {
          __builtin_memcpy(out + i, &w, sizeof(w));
        } else {
          T e[8];
          __builtin_memcpy(e, &w, sizeof(w));
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (j < left) out[i + j] = e[j];
        }
      } else {
        const uint32_t gone = (touched[u] | ~ok[u] | 0xffu << left) & 0xff;
        if (gone) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = (gone >> j) & 1 ? SPEC_NEG_INF : v[j];
        }
        float m = v[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) m = fmaxf(m, v[j]);
        if (m > bv) {   // (a thread meets its chunks in increasing order: the first maximum stays; NaN is never larger)
          bv = m;
#pragma unroll
          for (int j = 7; j >= 0; --j)
            if (v[j] == m) bi = i + j;
        }
      }
    }
    if (i0 - tid * 8 + kRowThreads * 8 * kRowChunks < V) load(i0 + kRowThreads * 8 * kRowChunks);
  }

  // ---- touched tokens (where logits and out are the same memory, these are still what they were) ----
  auto touch = [&](int i, int c, bool bit) {
#pragma unroll
    for (int j = 0; j < kMaxStages; ++j) c += j < n_path && path[j] == i;
    float v;
    if constexpr (BF16) v = bf16_bits_to_f32(row[i]);
    else v = row[i];
    v = penalized(v, i, c, bit, pen);
    if constexpr (OUT) {
      if constexpr (BF16) out[i] = (uint16_t)f32_to_bf16_bits(v);
      else out[i] = v;
    } else if (v > SPEC_NEG_INF && before(v, i, bv, bi)) {
      bv = v;
      bi = i;
    }
  };
  if (OUT) __syncthreads();
  if (pen.seen || pen.counts)
    for (int w = tid; w < n_words; w += kRowThreads) {
      uint32_t bits = 0;
      if (pen.seen) {
        bits = pen.seen[w];
        if (w * 32 + 32 > V) bits &= (1u << (V - w * 32)) - 1;
      } else {
        for (int j = 0; j < 32 && w * 32 + j < V; ++j) bits |= pen.counts[w * 32 + j] ? 1u << j : 0u;
      }
      while (bits) {
        const int i = w * 32 + __builtin_ctz(bits);
        bits &= bits - 1;
        touch(i, pen.counts ? pen.counts[i] : 0, pen.seen != nullptr);
      }
    }
  if (tid < n_path) {
    const int i = s_path[tid];
    bool first = (unsigned)i < (unsigned)V;
    for (int j = 0; j < tid; ++j) first = first && s_path[j] != i;
    if (first && !(pen.seen ? (pen.seen[i >> 5] >> (i & 31)) & 1 : pen.counts ? pen.counts[i] != 0 : 0)) touch(i, 0, false);
  }
  if (OUT) return;
  block_best<kRowThreads>(bv, bi, sv, si);
  if (tid == 0) p.greedy[blockIdx.x] = bi == kIdxNone ? 0 : bi;
}

hipError_t launch_logits(const LogitsJob& job, bool bf16, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)job.batch * (job.M + 1))), block(kRowThreads);
  const size_t smem = job.node_tok ? 2 * (size_t)job.M * sizeof(int32_t) : 0;
  if (job.out) {
    if (bf16) hipLaunchKernelGGL((logits_kernel<true, true>), grid, block, smem, st, job);
    else hipLaunchKernelGGL((logits_kernel<false, true>), grid, block, smem, st, job);
  } else {
    if (bf16) hipLaunchKernelGGL((logits_kernel<true, false>), grid, block, smem, st, job);
    else hipLaunchKernelGGL((logits_kernel<false, false>), grid, block, smem, st, job);
  }
  return hipGetLastError();
}

// One wave per sequence.  Position p of candidate c is predicted by the row of its prefix of length p: row 0, or the row of
// the node cand_node[c][p - 1].
__global__ __launch_bounds__(64) void accept_tree_kernel(AcceptTreeJob p) {
  const int q = blockIdx.x, lane = threadIdx.x, n = p.n, R = p.M + 1;
  const int nodes = p.n_nodes ? min(max(p.n_nodes[q], -1), p.M) : p.M;
  const int nc = p.n_cand ? p.n_cand[q] : p.B;
  const int32_t* greedy = p.greedy + (int64_t)q * R;
  const int32_t* cand = p.cand + (int64_t)q * p.B * n;
  const int32_t* node = p.cand_node + (int64_t)q * p.B * n;
  int32_t* out = p.out_tokens + (int64_t)q * (n + 1);
  int32_t* path = p.path_row + (int64_t)q * (n + 1);
  if (nodes < 0) {
    for (int c = lane; c < p.B; c += 64)
      if (p.accept_all) p.accept_all[(int64_t)q * p.B + c] = 0;
    if (lane <= n) out[lane] = path[lane] = -1;
    if (lane == 0) p.accept_len[q] = p.best_cand[q] = p.n_out[q] = 0;
    return;
  }
  float bv = -1.f;   // (accepted length, candidate): longer first, then smaller candidate index
  int32_t bi = kIdxNone;
  for (int c = lane; c < p.B; c += 64) {
    int32_t t[kMaxStages], row[kMaxStages];
#pragma unroll
    for (int i = 0; i < kMaxStages; ++i) {
      t[i] = i < n ? cand[c * n + i] : -1;
      row[i] = i == 0 ? 0 : i < n ? node[c * n + i - 1] + 1 : 0;
    }
    int a = 0;
    bool run = c < nc;
#pragma unroll
    for (int i = 0; i < kMaxStages; ++i) {
      // the token's own row has to be one of the sequence's: the bonus token is read from it
      const int own = i < n ? node[c * n + i] : -1;
      run = run && i < n && (unsigned)row[i] <= (unsigned)nodes && (unsigned)own < (unsigned)nodes;
      if (run) run = greedy[row[i]] == t[i];
      a += run ? 1 : 0;
    }
    if (p.accept_all) p.accept_all[(int64_t)q * p.B + c] = a;
    if (c < max(nc, 1) && before((float)a, c, bv, bi)) { bv = (float)a; bi = c; }
  }
  wave_best(bv, bi);
  const int a = (int)bv, best = bi;
  if (lane == 0) {
    p.accept_len[q] = a;
    p.best_cand[q] = best;
    p.n_out[q] = a + 1;
  }
  if (lane <= n) {
    const int row = lane == 0 ? 0 : lane <= a ? node[best * n + lane - 1] + 1 : -1;
    const int tok = lane < a ? cand[best * n + lane] : lane == a ? greedy[row] : -1;
    path[lane] = row;
    out[lane] = tok;
    // (whole numbers: their order does not matter)
    if (lane <= a && (unsigned)tok < (unsigned)p.V) {
      if (p.counts) atomicAdd(&p.counts[(int64_t)q * p.V + tok], 1);
      if (p.seen) atomicOr(&p.seen[(int64_t)q * ((p.V + 31) / 32) + (tok >> 5)], 1u << (tok & 31));
    }
  }
}

hipError_t launch_accept_tree(const AcceptTreeJob& job, hipStream_t st) {
  hipLaunchKernelGGL(accept_tree_kernel, dim3(job.batch), dim3(64), 0, st, job);
  return hipGetLastError();
}

}  // namespace specdraft
