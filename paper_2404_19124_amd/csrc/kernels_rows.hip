// The logits of a token tree's rows: penalties, biases and masks, the first maximum of every row, and the path of nodes
// that the base model agrees with.
//   c = counts[t] + occurrences of t on the row's path;  seen = its bit, or c > 0
//   v = logits[t];  seen: v = v > 0 ? v / repetition : v * repetition;  v -= frequency * c;  c > 0: v -= presence;
//   v += bias[t];  not allowed: v = -inf
#include <type_traits>

#include "device_utils.h"
#include "row_penalty.h"
#include "rows_internal.h"
#include "spec_internal.h"

namespace specdraft {

constexpr int row_chunks(bool out) { return out ? 1 : 2; }   // chunks of 8 tokens that a thread has in flight
// Up to so many rows have 1024 threads each, in more 512.  A verification of rows of 32000 with 1024 and with 512: 34 float32 rows 13.5
// and 16.4 us, 256 rows 19.3 and 22.3; from 280 to 500, where two rows share a CU (bfloat16) or take turns (float32: 120 KiB of LDS
// each), 25.9 to 30.2 and 26.4 to 29.3, alike; 650 bfloat16 rows 32.4 and 25.4, float32 38.2 and 40.5.
constexpr int kWideRows = 512;

// One workgroup per row, or (OUT, few rows) per `span` tokens of a row.  Few tokens of a row were seen or are on its path: TOUCHED
// tokens, and with them the last V % 8.  The others only take a bias and a mask, eight at a time, all loads of a trip requested a
// trip ahead.  The touched ones are left out there (their logits stay as they are): every wave lists their chunks, logits and all,
// and works 64 of them off at a time.  Consecutive rows run on one XCD, in whose L2 their sequence's counts stay, and the logits
// go past it: 2000 counts lie in half of a row's lines.
// Bound by reading the logits: 32 sequences of 45 rows of 128256 bf16 logits, 2000 tokens emitted, 379 MB in 116 us (3.3 TB/s;
// torch's largest sum reads 4.0 TB/s).  One element after the other: 603 us; touched tokens gathered again at a row's end: 140 us;
// rows dealt out over the XCDs one by one: 144 us.
template <bool BF16, bool OUT, int NT>
__global__ __launch_bounds__(NT, 4) void logits_kernel(LogitsJob p, int span) {
  typedef uint32_t words __attribute__((ext_vector_type(BF16 ? 4 : 8)));
  typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
  typedef float floatx8 __attribute__((ext_vector_type(8)));
  typedef typename std::conditional<BF16, uint16_t, float>::type T;
  typedef words loose __attribute__((aligned(sizeof(T))));   // (rows of an odd length start anywhere)
  constexpr int CHUNKS = row_chunks(OUT), STEP = NT * 8, TRIP = STEP * CHUNKS;
  constexpr int LIST = 64 * CHUNKS + 64;   // of a wave: a trip adds at most 64 * CHUNKS and finds at most 64 there
  struct Entry {
    uint32_t chunk, bits;   // its place in the row, / 8; touched tokens, from bit 8 on those that were seen, from 16 on those that are allowed
  };
  union Shared {
    words raw[NT / 64][LIST];
    int32_t node[2 * kMaxTreeItems];   // before the list: parents, tokens [M]
  };
  __shared__ __attribute__((aligned(32))) Shared s;
  __shared__ Entry s_list[NT / 64][LIST];
  auto& s_raw = s.raw;
  int32_t* s_node = s.node;
  __shared__ float sv[16];
  __shared__ int32_t si[16];
  __shared__ int32_t s_path[kMaxStages];
  __shared__ int s_n;
  const int R = p.M + 1, me = (int)(blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8), q = me / R, r = me - q * R, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = p.V;
  if (q >= p.batch) return;
  const int nodes = p.n_nodes ? min(max(p.n_nodes[q], -1), p.M) : p.M;
  if (r > nodes) {
    if (!OUT && tid == 0) p.greedy[me] = -1;
    return;
  }
  const T* row = static_cast<const T*>(p.logits) + (int64_t)me * V;
  T* out = OUT ? static_cast<T*>(p.out) + (int64_t)me * V : nullptr;
  const int begin = OUT ? (int)blockIdx.y * span : 0, end = OUT ? min(V, begin + span) : V, full = end & ~7;
  const RowPenalty pen = penalty_of(p.pen, q, me, V);

  words x[CHUNKS];
  uint32_t was_seen[CHUNKS] = {}, ok[CHUNKS];
  auto load = [&](int i0) {   // (lanes behind the last chunk read it again)
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) x[u] = __builtin_nontemporal_load(reinterpret_cast<const loose*>(row + min(i0 + u * STEP, full - 8)));
    if (pen.seen) {
#pragma unroll
      for (int u = 0; u < CHUNKS; ++u) was_seen[u] = reinterpret_cast<const uint8_t*>(pen.seen)[min(i0 + u * STEP, full - 8) >> 3];
    }
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) ok[u] = 0xff;
    if (pen.allowed) {
#pragma unroll
      for (int u = 0; u < CHUNKS; ++u) ok[u] = reinterpret_cast<const uint8_t*>(pen.allowed)[min(i0 + u * STEP, full - 8) >> 3];
    }
  };
  if (full > begin) load(begin + tid * 8);

  // ---- the tokens on the row's path ----
  int n_path = 0;
  if (p.node_tok && r > 0) {
    for (int i = tid; i < r; i += NT) {
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

  float bv = SPEC_NEG_INF;
  int32_t bi = kIdxNone;
  int listed = 0;   // chunks in the wave's list
  // the last chunks of the list, at most 64
  auto work_off = [&] {
    const int n = min(listed, 64);
    listed -= n;
    if (lane >= n) return;
    const Entry e = s_list[wave][listed + lane];
    for (uint32_t bits = e.bits & 0xff; bits; bits &= bits - 1) {
      const int j = __builtin_ctz(bits), i = (int)(e.chunk * 8) + j;
      const bool bit = (e.bits >> (8 + j)) & 1;
      int c = 0;
      float bias = 0.0f;
      if (pen.bias) bias = pen.bias[i];
      if (pen.counts && (bit || !pen.seen)) c = pen.counts[i];
      float v = to_f32(reinterpret_cast<const T*>(&s_raw[wave][listed + lane])[j]);
#pragma unroll
      for (int k = 0; k < kMaxStages; ++k) c += k < n_path && path[k] == i;
      v = penalized(v, c, bit, bias, (e.bits >> (16 + j)) & 1, pen);
      if constexpr (OUT) {
        if constexpr (BF16) out[i] = (uint16_t)f32_to_bf16_bits(v);
        else out[i] = v;
      } else if (v > SPEC_NEG_INF && before(v, i, bv, bi)) {
        bv = v;
        bi = i;
      }
    }
  };
  if (wave == 0 && end > full) {
    T e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = full + j < end ? row[full + j] : T(0);
    s_raw[0][0] = load_words<words>(e);
    uint32_t bits = ((1u << (end - full)) - 1) | 0xff0000;
    if (pen.seen) bits |= (uint32_t)reinterpret_cast<const uint8_t*>(pen.seen)[full >> 3] << 8;
    if (pen.allowed) bits &= 0xffff | (uint32_t)reinterpret_cast<const uint8_t*>(pen.allowed)[full >> 3] << 16;
    s_list[0][0] = {(uint32_t)full >> 3, bits};
    listed = 1;
  }
  for (int i0 = begin + tid * 8; i0 - tid * 8 < full; i0 += TRIP) {
    uint32_t touched[CHUNKS], seen[CHUNKS], allow[CHUNKS];
    words now[CHUNKS];
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) touched[u] = seen[u] = was_seen[u], allow[u] = ok[u], now[u] = x[u];
    if (i0 - tid * 8 + TRIP < full) load(i0 + TRIP);
    if (pen.counts && !pen.seen) {
#pragma unroll
      for (int u = 0; u < CHUNKS; ++u) {
        const i32x8 c = load_words<i32x8>(pen.counts + min(i0 + u * STEP, full - 8));
        touched[u] = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) touched[u] |= c[j] ? 1u << j : 0u;
      }
    }
    const uint32_t first = (uint32_t)__builtin_amdgcn_readfirstlane(i0 - lane * 8);
#pragma unroll
    for (int j = 0; j < kMaxStages; ++j) {
      // the wave's 512 tokens of a chunk hold it: one lane's eight do
      const uint32_t at = (uint32_t)path[j] - first;
      if (j < n_path && at < (uint32_t)TRIP && at % STEP < 512u) {
#pragma unroll
        for (int u = 0; u < CHUNKS; ++u) touched[u] |= at / STEP == (uint32_t)u && lane == (int)(at % STEP >> 3) ? 1u << (at & 7) : 0u;
      }
    }
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) {
      const bool mine = touched[u] && i0 + u * STEP < full;
      const uint64_t all = __ballot(mine);
      if (mine) {
        const int at = listed + __popcll(all & ((1ull << lane) - 1));
        s_raw[wave][at] = now[u];
        s_list[wave][at] = {(uint32_t)(i0 + u * STEP) >> 3, touched[u] | seen[u] << 8 | allow[u] << 16};
      }
      listed += __popcll(all);
    }
#pragma unroll
    for (int u = 0; u < CHUNKS; ++u) {
      const int i = i0 + u * STEP;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if constexpr (BF16) v[j] = bf16_bits_to_f32((uint16_t)(now[u][j / 2] >> (j & 1) * 16));
        else v[j] = __uint_as_float(now[u][j]);
      }
      if (pen.bias) {
        const floatx8 y = load_words<floatx8>(pen.bias + min(i, full - 8));
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = OUT && ((touched[u] >> j) & 1) ? v[j] : v[j] + y[j];
      }
      if constexpr (OUT) {
        const uint32_t gone = ~allow[u] & ~touched[u] & 0xff;
        if (gone) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = (gone >> j) & 1 ? SPEC_NEG_INF : v[j];
        }
        if (i >= full || (!pen.bias && !gone && p.out == p.logits)) continue;
        words w;
        if constexpr (BF16) {
#pragma unroll
          for (int j = 0; j < 4; ++j) w[j] = f32_to_bf16_pair(v[2 * j], v[2 * j + 1]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[j]);
        }
        __builtin_memcpy(out + i, &w, sizeof(w));
      } else {
        const uint32_t gone = i < full ? (touched[u] | ~allow[u]) & 0xff : 0xffu;
        if (gone) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = (gone >> j) & 1 ? SPEC_NEG_INF : v[j];
        }
        float m = v[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) m = fmaxf(m, v[j]);
        if (m >= bv && m > SPEC_NEG_INF) {   // (NaN is not)
          int32_t c = i;
#pragma unroll
          for (int j = 7; j >= 0; --j)
            if (v[j] == m) c = i + j;
          if (m > bv || c < bi) bi = c;
          bv = m;
        }
      }
    }
    while (listed > 64) work_off();
  }
  if (listed) work_off();
  if (OUT) return;
  block_best<NT>(bv, bi, sv, si);
  if (tid == 0) p.greedy[me] = bi == kIdxNone ? 0 : bi;
}

hipError_t launch_logits(const LogitsJob& job, bool bf16, hipStream_t st) {
  const int64_t rows = (int64_t)job.batch * (job.M + 1);
  const unsigned gx = (unsigned)(rows + 7) & ~7u;
  if (job.out) {   // parts of a row where there are few: 64 rows of 32003 whole: 21 us, in eight: 8 us
    const int parts = (int)min((int64_t)(job.V + 4095) / 4096, (1023 + rows) / rows), span = ((job.V + parts - 1) / parts + 31) & ~31;
    const dim3 grid(gx, (unsigned)((job.V + span - 1) / span));
    if (bf16) hipLaunchKernelGGL((logits_kernel<true, true, 512>), grid, dim3(512), 0, st, job, span);
    else hipLaunchKernelGGL((logits_kernel<false, true, 512>), grid, dim3(512), 0, st, job, span);
  } else if (rows <= kWideRows) {
    if (bf16) hipLaunchKernelGGL((logits_kernel<true, false, 1024>), dim3(gx), dim3(1024), 0, st, job, 0);
    else hipLaunchKernelGGL((logits_kernel<false, false, 1024>), dim3(gx), dim3(1024), 0, st, job, 0);
  } else {
    if (bf16) hipLaunchKernelGGL((logits_kernel<true, false, 512>), dim3(gx), dim3(512), 0, st, job, 0);
    else hipLaunchKernelGGL((logits_kernel<false, false, 512>), dim3(gx), dim3(512), 0, st, job, 0);
  }
  return hipGetLastError();
}

// One wave per sequence.  Position p of candidate c is predicted by the row of its prefix of length p: row 0, or the row of
// the node cand_node[c][p - 1].  Bound by latency, three loads one after the other: 4 us for 32 sequences of 16 candidates.
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
