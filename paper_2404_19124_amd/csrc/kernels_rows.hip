// The logits of a token tree's rows: penalties, biases and masks, the first maximum of every row, and the path of nodes
// that the base model agrees with.
//   c = counts[t] + occurrences of t on the row's path;  seen = its bit, or c > 0
//   v = logits[t];  seen: v = v > 0 ? v / repetition : v * repetition;  v -= frequency * c;  c > 0: v -= presence;
//   v += bias[t];  not allowed: v = -inf
#include "device_utils.h"
#include "rows_internal.h"
#include "spec_internal.h"

namespace specdraft {

constexpr int kRowThreads = 512;

// One workgroup per row.
template <bool BF16, bool OUT>
__global__ __launch_bounds__(kRowThreads) void logits_kernel(LogitsJob p) {
// (a product and a difference are rounded one by one: what is chosen must not hang on the compiler's choice)
#pragma clang fp contract(off)
  extern __shared__ int32_t s_parent[];   // [M]
  __shared__ float sv[16];
  __shared__ int32_t si[16];
  __shared__ int32_t s_path[kMaxStages];
  __shared__ int s_n;
  const int R = p.M + 1, q = blockIdx.x / R, r = blockIdx.x - q * R, tid = threadIdx.x;
  const int nodes = p.n_nodes ? min(max(p.n_nodes[q], -1), p.M) : p.M;
  if (r > nodes) {
    if (!OUT && tid == 0) p.greedy[blockIdx.x] = -1;
    return;
  }
  // the tokens on the row's path
  if (tid == 0) s_n = 0;
  if (p.node_tok) {
    for (int i = tid; i < r; i += kRowThreads) s_parent[i] = p.node_parent[(int64_t)q * p.M + i];
    __syncthreads();
    if (tid == 0) {
      int n = 0;
      for (int node = r - 1; node >= 0 && n < kMaxStages;) {
        s_path[n++] = p.node_tok[(int64_t)q * p.M + node];
        const int up = s_parent[node];
        node = up < node ? up : -1;
      }
      s_n = n;
    }
  }
  __syncthreads();
  const int n_path = s_n;
  const int words = (p.V + 31) / 32;
  const int32_t* counts = p.pen.counts ? p.pen.counts + (int64_t)q * p.V : nullptr;
  const uint32_t* seen = p.pen.seen ? p.pen.seen + (int64_t)q * words : nullptr;
  const float rep = p.pen.repetition ? p.pen.repetition[q] : 1.0f, pres = p.pen.presence ? p.pen.presence[q] : 0.0f;
  const float freq = p.pen.frequency ? p.pen.frequency[q] : 0.0f;
  const int bias_row = p.pen.bias ? p.pen.bias_row[q] : -1, mask_row = p.pen.allowed ? p.pen.mask_row[blockIdx.x] : -1;
  const float* bias = bias_row >= 0 && bias_row < p.pen.n_bias ? p.pen.bias + (int64_t)bias_row * p.V : nullptr;
  const uint32_t* allowed = mask_row >= 0 && mask_row < p.pen.n_allowed ? p.pen.allowed + (int64_t)mask_row * words : nullptr;
  const int64_t base = (int64_t)blockIdx.x * p.V;
  float bv = SPEC_NEG_INF;
  int32_t bi = kIdxNone;
  for (int i = tid; i < p.V; i += kRowThreads) {
    float v = BF16 ? bf16_bits_to_f32(static_cast<const uint16_t*>(p.logits)[base + i]) : static_cast<const float*>(p.logits)[base + i];
    const bool bit = seen ? (seen[i >> 5] >> (i & 31)) & 1 : false;
    int c = counts && (bit || !seen) ? counts[i] : 0;
    for (int j = 0; j < n_path; ++j) c += s_path[j] == i;
    if (bit || c > 0) v = v > 0.0f ? v / rep : v * rep;
    v = v - freq * (float)c;
    if (c > 0) v = v - pres;
    if (bias) v = v + bias[i];
    if (allowed && !((allowed[i >> 5] >> (i & 31)) & 1)) v = SPEC_NEG_INF;
    if (OUT) {
      if (BF16) static_cast<uint16_t*>(p.out)[base + i] = (uint16_t)f32_to_bf16_bits(v);
      else static_cast<float*>(p.out)[base + i] = v;
    } else if (v > bv) {   // (a thread meets its elements in increasing order: the first maximum stays)
      bv = v;
      bi = i;
    }
  }
  if (OUT) return;
  block_best<kRowThreads>(bv, bi, sv, si);
  if (tid == 0) p.greedy[blockIdx.x] = bi == kIdxNone ? 0 : bi;
}

hipError_t launch_logits(const LogitsJob& job, bool bf16, hipStream_t st) {
  const dim3 grid((unsigned)((int64_t)job.batch * (job.M + 1))), block(kRowThreads);
  const size_t smem = job.node_tok ? (size_t)job.M * sizeof(int32_t) : 0;
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
