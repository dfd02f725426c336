// The cache that spec_tree_attention reads: which blocks a sequence holds, where its next tokens go, and the copy of
// their keys and values into those slots.
#include "device_utils.h"
#include "rows_internal.h"
#include "spec_internal.h"

namespace specdraft {

// sums of 65535 demands of up to 2^30 tokens
__device__ __forceinline__ uint64_t wave_scan(uint64_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint64_t y = __shfl_up((unsigned long long)x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// blocks that `len` tokens need
__device__ __forceinline__ int blocks_of(int len, int size) { return (int)(((uint32_t)len + (uint32_t)size - 1) / (uint32_t)size); }

// (The two kernels of a large call: 48 sequences, prompts of 6000 tokens: 5 and 7 us, latency and the slot map's divisions.)
// One workgroup: prefix sums over the batch of the blocks and rows that are asked for.  A sequence is served while both sums
// fit, so the served ones come before the first that is not, and a sequence's share starts where the sum before it ends.
__global__ __launch_bounds__(1024) void extend_plan_kernel(ExtendJob p) {
  __shared__ uint64_t part[3][16];
  __shared__ unsigned long long s_fit[2];   // blocks and rows of the served ones: the sums in front of the first that is not
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int head = min(max(p.ring_state[0], 0), p.n_blocks - 1), count = min(max(p.ring_state[1], 0), p.n_blocks);
  const int limit = p.max_blocks * p.block_size;
  if (tid < 2) s_fit[tid] = ~0ull;
  uint64_t carry[3] = {0, 0, 0};
  for (int q0 = 0; q0 < p.batch; q0 += 1024) {
    const int q = q0 + tid;
    uint64_t x[3] = {0, 0, 0};   // blocks and rows asked for, blocks given back
    int old = 0, a = 0;
    if (q < p.batch) {
      old = min(max(p.ctx_len[q], 0), limit);
      a = p.add[q];
      if (a > limit - old) a = 0;
      if (a < -old) a = -old;
      const int have = blocks_of(old, p.block_size), want = blocks_of(old + a, p.block_size);
      if (a > 0) x[0] = want - have, x[1] = a;
      else x[2] = have - want;
    }
    uint64_t sum[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) sum[i] = wave_scan(x[i]);
    __syncthreads();   // the last round's sums have been read; s_fit is set
    if (lane == 63)
#pragma unroll
      for (int i = 0; i < 3; ++i) part[i][wave] = sum[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      uint64_t before = carry[i];
      for (int w = 0; w < 16; ++w) {
        if (w < wave) before += part[i][w];
        carry[i] += part[i][w];
      }
      sum[i] += before;
    }
    const bool served = a <= 0 || (sum[0] <= (uint64_t)count && sum[1] <= (uint64_t)p.cap);
    if (!served) {
      atomicMin(&s_fit[0], (unsigned long long)(sum[0] - x[0]));
      atomicMin(&s_fit[1], (unsigned long long)(sum[1] - x[1]));
    }
    __syncthreads();
    if (q < p.batch) {
      p.new_len[q] = served ? old + a : old;
      p.added[q] = served ? a : 0;
      p.row_start[q] = (int32_t)min((uint64_t)s_fit[1], sum[1] - x[1]);
    }
  }
  if (tid == 0) {
    const uint64_t taken = min((uint64_t)s_fit[0], carry[0]);
    p.row_start[p.batch] = (int32_t)min((uint64_t)s_fit[1], carry[1]);
    p.ring_state_new[0] = (int32_t)(((uint64_t)head + taken) % (uint64_t)p.n_blocks);
    p.ring_state_new[1] = (int32_t)min((uint64_t)count - taken + carry[2], (uint64_t)p.n_blocks);
  }
}

// Workgroup (x, y) carries out the shares of the x-th stretch of sequences one after the other, each strided over y; the ones behind
// the last stretch mark the entries behind the last token.  Where the stretch's shares start in the ring is summed up once more from
// the lengths: a few words from the cache, and no workspace.  Reads and writes of the ring do not meet: what is taken lies among its
// `count` entries, what is given back goes behind them.
// (A workgroup per sequence sums up the whole batch each time: 65535 sequences 143 ms, in stretches of 64 0.6 ms.)
__global__ __launch_bounds__(256) void extend_fill_kernel(ExtendJob p, int stretch) {
  __shared__ uint64_t part[4][4];
  const int tid = threadIdx.x, at = blockIdx.y * 256 + tid, step = gridDim.y * 256;
  if (blockIdx.x == gridDim.x - 1) {
    for (int t = p.row_start[p.batch] + at; t < p.cap; t += step) {
      p.slot[t] = -1;
      if (p.pos) p.pos[t] = -1;
      if (p.path_row) p.src_row[t] = -1;
    }
    return;
  }
  const int first_q = blockIdx.x * stretch, last_q = min(first_q + stretch, p.batch);
  int a = p.added[first_q], now = p.new_len[first_q], first = p.row_start[first_q];   // (requested ahead)
  uint64_t sum[4] = {0, 0, 0, 0};   // blocks taken and given back: before the next sequence, by all
  for (int i = tid; i < p.batch; i += 256) {
    const int d = p.added[i], now = p.new_len[i];
    const int change = blocks_of(now, p.block_size) - blocks_of(now - d, p.block_size);
    sum[2] += max(change, 0);
    sum[3] += max(-change, 0);
    if (i < first_q) sum[0] += max(change, 0), sum[1] += max(-change, 0);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sum[i] = wave_scan(sum[i]);
    if ((tid & 63) == 63) part[i][tid >> 6] = sum[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = part[i][0] + part[i][1] + part[i][2] + part[i][3];
  const uint64_t n = p.n_blocks;
  // (the ring before this call)
  const uint64_t head = ((uint64_t)p.ring_state_new[0] + n - sum[2] % n) % n;
  const uint64_t count = (uint64_t)p.ring_state_new[1] + sum[2] - sum[3];
  for (int q = first_q;;) {
    const int old = now - a;
    const int have = blocks_of(old, p.block_size), want = blocks_of(now, p.block_size);
    int32_t* row = p.block_table + (int64_t)q * p.max_blocks;
    for (int i = want + at; i < have; i += step) p.ring[(head + count + sum[1] + (uint64_t)(i - want)) % n] = row[i];
    for (int i = have + at; i < want; i += step) row[i] = p.ring[(head + sum[0] + (uint64_t)(i - have)) % n];
    for (int j = at; j < a; j += step) {
      const int t = old + j, b = t / p.block_size;
      // (a new block's entry may be under way to the table)
      const int block = b < have ? row[b] : p.ring[(head + sum[0] + (uint64_t)(b - have)) % n];
      p.slot[first + j] = block >= 0 && block < p.n_blocks ? block * p.block_size + t % p.block_size : -1;
      if (p.pos) p.pos[first + j] = t;
      if (p.path_row) {
        const int r = j < p.path_width ? p.path_row[(int64_t)q * p.path_width + j] : -1;
        p.src_row[first + j] = r >= 0 && r < p.seq_rows ? q * p.seq_rows + r : -1;
      }
    }
    sum[0] += (uint64_t)max(want - have, 0);
    sum[1] += (uint64_t)max(have - want, 0);
    if (++q == last_q) return;
    a = p.added[q], now = p.new_len[q], first = p.row_start[q];
  }
}

__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

// Both in one, for a step of decoding: one workgroup, a sequence per thread, then an entry of the slot map per thread, whose
// sequence is searched for among the shares' starts, and a wave per sequence that gives blocks back.  Bound by latency alone, replayed: 64
// sequences and 192 entries take 5.9 us, the two kernels 9.8 us; 1920 entries 7.3 and 9.8 us, 8000 entries 12.9 and 9.9 us.
constexpr int kOneBatch = 1024, kOneCap = 4096;
__global__ __launch_bounds__(kOneBatch) void extend_kernel(ExtendJob p) {
  __shared__ uint32_t part[2][16], s_fit[2], s_rows[kOneBatch], s_blocks[kOneBatch];
  __shared__ uint64_t back[16], s_back[kOneBatch];
  __shared__ int s_old[kOneBatch], s_added[kOneBatch];
  const int q = threadIdx.x, lane = q & 63, wave = q >> 6;
  const int head = min(max(p.ring_state[0], 0), p.n_blocks - 1), count = min(max(p.ring_state[1], 0), p.n_blocks);
  const int limit = p.max_blocks * p.block_size;
  // blocks and rows asked for (a demand past the slot map's end is not served, how far past does not matter), blocks given back
  uint32_t x[2] = {0, 0}, sum[2];
  uint64_t x_back = 0;
  int old = 0, a = 0;
  if (q < p.batch) {
    old = min(max(p.ctx_len[q], 0), limit);
    a = p.add[q];
    if (a > limit - old) a = 0;
    if (a < -old) a = -old;
    const int have = blocks_of(old, p.block_size), want = blocks_of(old + a, p.block_size);
    if (a > 0) x[0] = (uint32_t)min(want - have, p.cap + 1), x[1] = (uint32_t)min(a, p.cap + 1);
    else x_back = (uint64_t)(have - want);
  }
  if (q < 2) s_fit[q] = ~0u;
#pragma unroll
  for (int i = 0; i < 2; ++i) sum[i] = wave_scan(x[i]);
  uint64_t sum_back = wave_scan(x_back);
  if (lane == 63) part[0][wave] = sum[0], part[1][wave] = sum[1], back[wave] = sum_back;
  __syncthreads();
  uint32_t all[2] = {0, 0};
  uint64_t all_back = 0;
  for (int w = 0; w < 16; ++w) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (w < wave) sum[i] += part[i][w];
      all[i] += part[i][w];
    }
    if (w < wave) sum_back += back[w];
    all_back += back[w];
  }
  const bool served = a <= 0 || (sum[0] <= (uint32_t)count && sum[1] <= (uint32_t)p.cap);
  if (!served) {
    atomicMin(&s_fit[0], sum[0] - x[0]);
    atomicMin(&s_fit[1], sum[1] - x[1]);
  }
  __syncthreads();
  const uint32_t taken = min(s_fit[0], all[0]);
  const int rows = (int)min(s_fit[1], all[1]);
  s_rows[q] = q < p.batch ? min(s_fit[1], sum[1] - x[1]) : 0x7fffffffu;
  s_blocks[q] = sum[0] - x[0];
  s_back[q] = sum_back - x_back;
  s_old[q] = old;
  s_added[q] = served ? a : 0;
  if (q < p.batch) {
    p.new_len[q] = served ? old + a : old;
    p.added[q] = served ? a : 0;
    p.row_start[q] = (int32_t)s_rows[q];
  }
  if (q == 0) {
    p.row_start[p.batch] = rows;
    p.ring_state_new[0] = (int32_t)(((uint64_t)head + taken) % (uint64_t)p.n_blocks);
    p.ring_state_new[1] = (int32_t)min((uint64_t)count - taken + all_back, (uint64_t)p.n_blocks);
  }
  __syncthreads();
  for (int t = q; t < p.cap; t += kOneBatch) {
    int slot = -1, pos = -1, src = -1;
    if (t < rows) {
      int of = 0;   // the last sequence whose share starts at or before t
#pragma unroll
      for (int step = kOneBatch / 2; step > 0; step /= 2)
        if (s_rows[of + step] <= (uint32_t)t) of += step;
      const int j = t - (int)s_rows[of], b = (s_old[of] + j) / p.block_size, in = s_old[of] + j - b * p.block_size;
      const int have = blocks_of(s_old[of], p.block_size);
      int32_t* entry = p.block_table + (int64_t)of * p.max_blocks + b;
      int block;
      if (b < have) {
        block = *entry;
      } else {
        block = p.ring[((uint32_t)head + s_blocks[of] + (uint32_t)(b - have)) % (uint32_t)p.n_blocks];
        if (in == 0) *entry = block;   // (every new block's first token is among the new ones)
      }
      pos = s_old[of] + j;
      if (block >= 0 && block < p.n_blocks) slot = block * p.block_size + in;
      if (p.path_row) {
        const int r = j < p.path_width ? p.path_row[(int64_t)of * p.path_width + j] : -1;
        if (r >= 0 && r < p.seq_rows) src = of * p.seq_rows + r;
      }
    }
    p.slot[t] = slot;
    if (p.pos) p.pos[t] = pos;
    if (p.path_row) p.src_row[t] = src;
  }
  for (int w = wave; w < p.batch; w += kOneBatch / 64) {
    if (s_added[w] >= 0) continue;
    const int have = blocks_of(s_old[w], p.block_size), want = blocks_of(s_old[w] + s_added[w], p.block_size);
    const int32_t* row = p.block_table + (int64_t)w * p.max_blocks;
    for (int i = want + lane; i < have; i += 64)
      p.ring[((uint64_t)head + (uint64_t)count + s_back[w] + (uint64_t)(i - want)) % (uint64_t)p.n_blocks] = row[i];
  }
}

hipError_t launch_extend(const ExtendJob& job, hipStream_t st) {
  if (job.batch <= kOneBatch && job.cap <= kOneCap) {
    hipLaunchKernelGGL(extend_kernel, dim3(1), dim3(kOneBatch), 0, st, job);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(extend_plan_kernel, dim3(1), dim3(1024), 0, st, job);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // at most kFillGroups workgroups, each of which reads the batch's lengths; up to 32 where a sequence may have many tokens
  constexpr int kFillGroups = 4096, kStretches = 1024;
  const int stretch = (job.batch + kStretches - 1) / kStretches, stretches = (job.batch + stretch - 1) / stretch;
  const int most = min(job.cap / 1024 + 1, min(32, kFillGroups / stretches));
  hipLaunchKernelGGL(extend_fill_kernel, dim3(stretches + 1, most), dim3(256), 0, st, job, stretch);
  return hipGetLastError();
}

// Copy of one 16-byte word of a token's keys and one of its values per thread and turn; neighbours copy neighbouring words of a
// row.  Bound by memory: 16000 rows of 8 heads of 128 in 8 layers, 1.05 GB, 187 us, 5.6 TB/s read and written; 3 rows of 32 heads
// in 32 layers 3 us, a launch.
__global__ __launch_bounds__(256) void store_kernel(StoreJob p) {
  const int per = p.kv_heads * p.row_words, layer = blockIdx.y;
  const int64_t total = (int64_t)p.count * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int t = (int)(i / per), w = (int)(i - (int64_t)t * per), h = w / p.row_words, c = w - h * p.row_words;
    const int slot = p.slot[t], src = p.src_row ? p.src_row[t] : t;
    if (slot < 0 || slot >= p.n_slots || src < 0 || src >= p.rows) continue;
    const int64_t from = layer * p.new_layer + src * p.new_row + h * p.new_head + c * 16;
    const int64_t to = layer * p.layer + slot / p.block_size * p.block + slot % p.block_size * p.slot_stride + h * p.head + c * 16;
    *reinterpret_cast<u32x4*>(p.k + to) = *reinterpret_cast<const u32x4*>(p.k_new + from);
    *reinterpret_cast<u32x4*>(p.v + to) = *reinterpret_cast<const u32x4*>(p.v_new + from);
  }
}

hipError_t launch_store(const StoreJob& job, hipStream_t st) {
  const int64_t words = (int64_t)job.count * job.kv_heads * job.row_words, groups = (words + 255) / 256;
  hipLaunchKernelGGL(store_kernel, dim3((unsigned)(groups < 4096 ? groups : 4096), job.layers), dim3(256), 0, st, job);
  return hipGetLastError();
}

}  // namespace specdraft
