// Attention of a token tree's rows over a paged cache and their own ancestors:
//   out[r][h] = sum_k softmax_k(scale * q[r][h] . key_k[g]) value_k[g],   g = h / (q_heads / kv_heads)
// over the cached tokens and the rows 0, the ancestors of r, and r.
#include "device_utils.h"
#include "rows_internal.h"
#include "spec_internal.h"

namespace specdraft {

template <bool BF16>
__device__ __forceinline__ float load_element(const uint8_t* at, int i) {
  if constexpr (BF16) return bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(at)[i]);
  else return reinterpret_cast<const float*>(at)[i];
}

// One workgroup per (row, query head, sequence): its four waves take every fourth key, four elements of a row per lane, with
// the running maximum and sum of the softmax, and are joined at the end.
template <bool BF16>
__global__ __launch_bounds__(256) void attention_kernel(AttentionJob p) {
  __shared__ float s_m[4], s_l[4], s_o[4][256];
  __shared__ int s_row[kMaxStages + 1], s_rows;
  const int r = blockIdx.x, h = blockIdx.y, q = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int nodes = p.n_nodes ? min(max(p.n_nodes[q], -1), p.M) : p.M;
  if (r > nodes) return;
  const int g = h / (p.q_heads / p.kv_heads), ctx = min(max(p.ctx_len[q], 0), p.max_blocks * p.block_size);
  if (tid == 0) {
    int n = 0;
    for (int node = r - 1; node >= 0 && n < kMaxStages;) {
      s_row[n++] = node + 1;
      const int up = p.node_parent[(int64_t)q * p.M + node];
      node = up < node ? up : -1;
    }
    s_row[n++] = 0;
    s_rows = n;
  }
  __syncthreads();
  const uint8_t* qr = static_cast<const uint8_t*>(p.q) + q * p.q_seq + r * p.q_row + h * p.q_head;
  float x[4], o[4] = {0, 0, 0, 0}, m = SPEC_NEG_INF, l = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = lane + i * 64 < p.head_dim ? load_element<BF16>(qr, lane + i * 64) * p.scale : 0.0f;
  const int keys = ctx + s_rows;
  for (int t = wave; t < keys; t += 4) {
    const uint8_t *k, *v;
    if (t < ctx) {
      const int b = p.block_table[(int64_t)q * p.max_blocks + t / p.block_size];
      if (b < 0 || b >= p.n_blocks) continue;
      const int64_t at = b * p.block + t % p.block_size * p.slot + g * p.cache_head;
      k = static_cast<const uint8_t*>(p.k) + at;
      v = static_cast<const uint8_t*>(p.v) + at;
    } else {
      const int64_t at = q * p.new_seq + s_row[t - ctx] * p.new_row + g * p.new_head;
      k = static_cast<const uint8_t*>(p.k_new) + at;
      v = static_cast<const uint8_t*>(p.v_new) + at;
    }
    float s = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + i * 64 < p.head_dim) s += x[i] * load_element<BF16>(k, lane + i * 64);
    s = wave_sum(s);
    const float top = fmaxf(m, s), w = expf(s - top), keep = expf(m - top);
    l = l * keep + w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + i * 64 < p.head_dim) o[i] = o[i] * keep + w * load_element<BF16>(v, lane + i * 64);
    m = top;
  }
  if (lane == 0) s_m[wave] = m, s_l[wave] = l;
#pragma unroll
  for (int i = 0; i < 4; ++i) s_o[wave][lane + i * 64] = o[i];
  __syncthreads();
  // (row 0 is always there: one of the four has a key)
  const float top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3]));
  float sum = 0, val = 0;
  for (int w = 0; w < 4; ++w) {
    const float f = expf(s_m[w] - top);
    sum += f * s_l[w];
    val += f * s_o[w][tid];
  }
  if (tid < p.head_dim) {
    uint8_t* to = static_cast<uint8_t*>(p.out) + q * p.out_seq + r * p.out_row + h * p.out_head;
    if constexpr (BF16) reinterpret_cast<uint16_t*>(to)[tid] = (uint16_t)f32_to_bf16_bits(val / sum);
    else reinterpret_cast<float*>(to)[tid] = val / sum;
  }
}

int64_t attention_workspace(int batch, int M, int q_heads, int kv_heads, int head_dim, bool bf16) { return 0; }

hipError_t launch_attention(const AttentionJob& job, bool bf16, hipStream_t st) {
  const dim3 grid(job.M + 1, job.q_heads, job.batch);
  if (bf16) hipLaunchKernelGGL((attention_kernel<true>), grid, dim3(256), 0, st, job);
  else hipLaunchKernelGGL((attention_kernel<false>), grid, dim3(256), 0, st, job);
  return hipGetLastError();
}

}  // namespace specdraft
