// Attention of a token tree's rows over a paged cache and their own ancestors:
//   out[r][h] = sum_k softmax_k(scale * q[r][h] . key_k[g]) value_k[g],   g = h / (q_heads / kv_heads)
// over the cached tokens and the rows 0, the ancestors of r, and r.
//
// A UNIT is BM query rows of one key/value head of one sequence: the rows of all query heads that share it, tree row by tree
// row.  Its keys are the cached tokens and then the sequence's rows, in TILES of 64.  One pass over the tiles keeps, per
// query row, a bound m of the scores so far, the sum l of the softmax's weights exp(score - m) and the weighted sum o of the
// values (with a larger bound m', l and o are multiplied by exp(m - m')).
//
// Bound by reading the keys and values, beyond the L2 as often as a head has blocks of rows, and by latency in small calls.  Replayed from
// a graph: 64 sequences of one token over up to 8000 (8 heads of 128, 64 query heads) 200 us, 5.0 TB/s; 48 of 33 rows over up to 2000
// (32 heads) 219 us, 4.7 TB/s; 32 of 45 rows over up to 4000 (8 heads, 64 query heads) 208 us, 570 TFLOP/s, 980 MB read for 385 of keys and
// values; one of 34 rows over 600 (32 heads) 15.9 us, 62 % of it waiting.  Scores are computed transposed, keys times queries, so that a lane's registers hold one query
// row's scores: the softmax, and the rescaling of the transposed sums, need no exchange but two swaps.  Weights are rounded to
// bfloat16 for the second product, each by at most 2^-8 of itself (a product in float32 has an eighth of the rate: 141 and 1153
// TFLOP/s), and their sum is that of the rounded ones: an output is a mean of the values with weights that far from the exact ones.
#include <atomic>

#include "attention_body.h"

namespace specdraft {

// How a workgroup copies tiles into LDS, one ahead of the one it works on, across its segments.  A wave copies a fourth of a
// tile's rows, 1 KiB (RPI rows) per instruction.  Where the wave's 16 tokens lie in one page, their place is one address for all
// lanes, and the lanes' offsets from it are the same for every tile: it is found for 64 tiles at once, a tile per lane.
// Otherwise (rows of the tree, the last cached tokens, pages of other sizes, blocks out of range) lane l finds the place of row
// l % 16.  (The second way for every tile: 154 vector instructions per tile instead of 30.)
template <bool BF16, int DP, int MQ, int WK>
struct TileCopy {
  typedef AttentionShape<BF16, DP, MQ, WK> S;
  static constexpr bool kEarly = false;        // a tile is requested when its buffer is free
  static constexpr int RW = KT / 4;
  static constexpr int RPI = 64 / S::CH;
  static constexpr int NL = RW / RPI;          // instructions for keys, and for values
  const AttentionJob& p;
  uint32_t (*s_valid)[4];
  int last_word;
  int64_t to_v_cache, to_v_rows;               // from a key to its value
  uint32_t offset[NL];                         // of this lane's words from the place of the wave's rows
  // for the segment that is worked on and for the one behind it: offsets into the cache of the wave's rows of 64 tiles from
  // tile `base` on (lane by lane, -1: no single place)
  struct Places {
    int64_t at;
    int base;
  };
  // the tile that is copied next, where it has no single place: this lane's offset from the head's keys in the cache, or (bit 0)
  // from those of the tree's rows, and which of the wave's rows are cached tokens
  struct Rows {
    uint64_t at;
    uint32_t valid;
  };

  static __device__ __forceinline__ void landed() { __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8)); }   // vmcnt(0)

  __device__ __forceinline__ void init() {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      const int row = j * RPI + lane / S::CH, word = (lane % S::CH) ^ ((wave * RW + row) & S::SWZ);
      offset[j] = (uint32_t)(row * (int)p.slot + min(word, last_word) * 16);
    }
  }

  __device__ __forceinline__ Places places(const Segment& s, int base) const {
    const int lane = threadIdx.x & 63, key = (s.tile0 + base + lane) * KT + (int)(threadIdx.x >> 6) * RW;
    Places r = {-1, base};
    if (p.one_place && key + RW <= s.ctx && base + lane < s.n_tiles) {
      const int b = key / p.block_size, x = p.block_table[(int64_t)s.q * p.max_blocks + b];
      if (x >= 0 && x < p.n_blocks) r.at = x * p.block + (key - b * p.block_size) * p.slot;
    }
    return r;
  }
  static __device__ __forceinline__ int64_t place_of(const Places& f, int t) {
    const int lane = t - f.base;
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(f.at >> 32), lane) << 32 |
                     (uint32_t)__builtin_amdgcn_readlane((int)f.at, lane));
  }

  __device__ __forceinline__ Rows rows_of(const Segment& s, int t) const {
    const int tid = opaque_tid(), key = (s.tile0 + t) * KT + (tid >> 6) * RW + (tid & 63) % RW;
    // what is not a key is read from row 0, which every row sees: with a weight of zero it adds nothing
    uint64_t a = 1;
    bool ok = false;
    if (key < s.ctx) {
      const int b = key / p.block_size, x = p.block_table[(int64_t)s.q * p.max_blocks + b];
      if (x >= 0 && x < p.n_blocks) {
        a = (uint64_t)(x * p.block + (key - b * p.block_size) * p.slot);
        ok = true;
      }
    } else if (key < s.keys) {
      a = (uint64_t)((key - s.ctx) * p.new_row) | 1;
    }
    return {a, (uint32_t)__ballot(ok) & ((1u << RW) - 1)};
  }

  // what copying a tile needs
  struct Source {
    uint64_t k_cache, k_rows;   // addresses of the head's; 0: nothing to copy
    int64_t place;              // -1: row by row
    Rows r;
  };
  static __device__ __forceinline__ Source nothing() { return {0, 0, 0, {0, 0}}; }
  // of tile t of a segment; called for its tiles one after the other
  __device__ __forceinline__ Source source(const Segment& s, int t, Places& f) const {
    if (t - f.base == 64) f = places(s, t);
    Source x = {reinterpret_cast<uint64_t>(s.k_cache), reinterpret_cast<uint64_t>(s.k_rows), place_of(f, t), {0, 0}};
    if (x.place < 0) x.r = rows_of(s, t);
    return x;
  }

  // (as buffer instructions: behind copies into LDS that go through flat addresses, the compiler waits for all LDS reads at once)
  __device__ __forceinline__ static void copy16(uint64_t from, uint32_t offset, lds_u8* to) {
    const auto place = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(uniform(from)), 0, -1, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(place, (__attribute__((address_space(3))) void*)to, 16, offset, 0, 0, 0);
  }
  // a lane's 16 bytes land at its place in the instruction's 1 KiB: the words of a row are permuted where they are read
  __device__ __forceinline__ void copy(const Source& s, lds_u8* to, uint32_t* valid) const {
    const int tid = opaque_tid(), lane = tid & 63, wave = uniform(tid >> 6);
    lds_u8* at = to + wave * RW * S::ROWB;
    if (s.place >= 0) {
      if (lane == 0) valid[wave] = (1u << RW) - 1;
      const uint64_t k = s.k_cache + s.place, v = k + to_v_cache;
#pragma unroll
      for (int j = 0; j < NL; ++j) {
        copy16(k, offset[j], at + j * RPI * S::ROWB);
        copy16(v, offset[j], at + (KT + j * RPI) * S::ROWB);
      }
      return;
    }
    if (lane == 0) valid[wave] = s.r.valid;
    const uint64_t k_cache = s.k_cache, k_rows = s.k_rows;
    if (p.offsets_fit) {
#pragma unroll
      for (int j = 0; j < NL; ++j) {
        const int row = j * RPI + lane / S::CH, word = min((lane % S::CH) ^ ((wave * RW + row) & S::SWZ), last_word);
        const uint32_t x = (uint32_t)__shfl((int)s.r.at, row), from = (x & ~1u) + word * 16;
        lds_u8 *k = at + j * RPI * S::ROWB, *v = at + (KT + j * RPI) * S::ROWB;
        if (x & 1) {
          copy16(k_rows, from, k);
          copy16(k_rows + to_v_rows, from, v);
        } else {
          copy16(k_cache, from, k);
          copy16(k_cache + to_v_cache, from, v);
        }
      }
      return;
    }
#pragma unroll 1
    for (int row = 0; row < RW; ++row) {   // (a cache of more than 4 GiB) row by row, by the lanes whose words are theirs
      const uint64_t x = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(s.r.at >> 32), row) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)s.r.at, row);
      const uint64_t k = (x & ~1ull) + (x & 1 ? k_rows : k_cache), v = k + (x & 1 ? to_v_rows : to_v_cache);
      const int word = (lane % S::CH) ^ ((wave * RW + row) & S::SWZ), j = row / RPI;
      if (lane / S::CH == row % RPI) {
        copy16(k, min(word, last_word) * 16, at + j * RPI * S::ROWB);
        copy16(v, min(word, last_word) * 16, at + (KT + j * RPI) * S::ROWB);
      }
    }
  }
};

template <bool BF16, int DP, int MQ, int WK>
__global__ __launch_bounds__(256, tile_bytes(KT * DP * (BF16 ? 2 : 4)) <= 65536 ? 2 : 1) void attention_kernel(AttentionJob p, AttentionSpace ws) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  __shared__ uint32_t s_valid[2][4], s_again;
  attention_body<BF16, DP, MQ, WK, TileCopy<BF16, DP, MQ, WK>>(p, ws, smem, s_valid, s_again);
}

// float32 heads of more than 128 elements (two buffers of their tiles do not fit a CU's memory with 64 keys): units of 16 query
// rows, four to a wave, straight from memory.  16 lanes take a key, four keys at once, 16 elements of the head per lane; the
// waves read the same keys, three of them from the cache.  Bound by the latency of a key's loads, one key ahead, and the vector
// units: 4 sequences of up to 1000 tokens, 32 query heads on 8 of 192, 32 rows: 320 us, 8.3 TFLOP/s; one of 20000 tokens, 8 query
// heads on one of 256: 117 us.  (A workgroup per row, unsplit: 1.02 ms and 12.1 ms.)
__global__ __launch_bounds__(256, 2) void attention_wide_kernel(AttentionJob p, AttentionSpace ws) {
  constexpr int BM = kWideRows, DP = 256;
  const int G = p.q_heads / p.kv_heads, tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l16 = lane & 15, grp = lane >> 4;
  Schedule<BM, unit_cost(false)> plan = {p, G};
  if (!plan.live(ws)) return;
  Segment now;
  Owner mine = {-1, 0, 0, 0, 0};
  bool more = plan.first(now);
  const float sc = p.scale * kLog2e;
  while (more) {
    const int rows = (now.nodes + 1) * G - now.block * BM;
    f32x4 x[4][4], o[4][4];
    float m[4], l[4];
    int row_of[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int mm = wave * 4 + i < rows ? now.block * BM + wave * 4 + i : now.block * BM;
      row_of[i] = mm / G;
      const float* from = reinterpret_cast<const float*>(static_cast<const uint8_t*>(p.q) + now.q * p.q_seq + (int64_t)row_of[i] * p.q_row +
                                                         (int64_t)(now.g * G + mm % G) * p.q_head);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int e = c * 64 + l16 * 4;
        x[i][c] = e < p.head_dim && p.scale != 0 ? *reinterpret_cast<const f32x4*>(from + e) : (f32x4){0, 0, 0, 0};
        o[i][c] = (f32x4){0, 0, 0, 0};
      }
      m[i] = kLowest, l[i] = 0;
    }
    const int64_t to_v_cache = static_cast<const uint8_t*>(p.v) - static_cast<const uint8_t*>(p.k);
    const int64_t to_v_rows = static_cast<const uint8_t*>(p.v_new) - static_cast<const uint8_t*>(p.k_new);
    auto load = [&](const uint8_t* at, f32x4 (&y)[4]) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int e = c * 64 + l16 * 4;
        y[c] = e < p.head_dim ? *reinterpret_cast<const f32x4*>(at + e * 4) : (f32x4){0, 0, 0, 0};
      }
    };
    auto take = [&](const f32x4 (&k)[4], const f32x4 (&v)[4], uint32_t sees) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 d = x[i][0] * k[0];
#pragma unroll
        for (int c = 1; c < 4; ++c) d += x[i][c] * k[c];
        const float score = row16_sum((d[0] + d[1]) + (d[2] + d[3])) * sc;
        if ((sees >> i) & 1) {
          if (score > m[i]) {
            const float keep = __builtin_amdgcn_exp2f(m[i] - (score + kSlack));
            m[i] = score + kSlack;
            l[i] *= keep;
#pragma unroll
            for (int c = 0; c < 4; ++c) o[i][c] *= keep;
          }
          const float w = __builtin_amdgcn_exp2f(score - m[i]);
          l[i] += w;
#pragma unroll
          for (int c = 0; c < 4; ++c) o[i][c] += w * v[c];
        }
      }
    };
    // ---- cached tokens: the next key's loads are sent before one is worked on ----
    const int from = now.tile0 * KT, to = min((now.tile0 + now.n_tiles) * KT, now.keys), cached = min(to, now.ctx);
    auto place = [&](int key) -> const uint8_t* {   // NULL: takes no part
      if (key >= cached) return nullptr;
      const int b = key / p.block_size, t = p.block_table[(int64_t)now.q * p.max_blocks + b];
      return t >= 0 && t < p.n_blocks ? now.k_cache + t * p.block + (key - b * p.block_size) * p.slot : nullptr;
    };
    f32x4 k[4], v[4];
    const uint8_t* at = place(from + grp);
    if (at) load(at, k), load(at + to_v_cache, v);
    for (int t = from; t < cached; t += 4) {
      const uint8_t* next = place(t + 4 + grp);
      f32x4 k2[4], v2[4];
      if (next) load(next, k2), load(next + to_v_cache, v2);
      if (at) take(k, v, 15);
      at = next;
#pragma unroll
      for (int c = 0; c < 4; ++c) k[c] = k2[c], v[c] = v2[c];
    }
    // ---- rows of the tree ----
    for (int t = max(from, now.ctx); t < to; t += 4) {
      const int r = t + grp - now.ctx;
      uint32_t sees = 0;
      if (t + grp < to) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          int row = row_of[i];
          for (int n = 0; n < kMaxStages && row > r; ++n) {
            const int up = p.node_parent[(int64_t)now.q * p.M + row - 1];
            row = n + 1 < kMaxStages && up >= 0 && up < row - 1 ? up + 1 : 0;
          }
          if (row == r) sees |= 1u << i;
        }
      }
      if (sees) {
        load(now.k_rows + (int64_t)r * p.new_row, k);
        load(now.k_rows + to_v_rows + (int64_t)r * p.new_row, v);
        take(k, v, sees);
      }
    }
    // ---- join of the four keys' lanes; lane group i writes row i ----
    const bool whole = now.n_seg == now.tiles;
    if (!whole && now.tile0 == 0) mine = {now.q, now.g, now.block, plan.last(), min(rows, BM)};
    f32x4 y[4];
    float top = 0, sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float all_m = groups_max(m[i]), f = __builtin_amdgcn_exp2f(m[i] - all_m), all_l = groups_sum(l[i] * f);
      if (grp == i) top = all_m, sum = all_l;
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float s = groups_sum(f > 0 ? o[i][c][j] * f : 0.0f);
          if (grp == i) y[c][j] = s;
        }
    }
    const int r = wave * 4 + grp;
    if (r < rows) {
      const int mm = now.block * BM + r;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int e = c * 64 + l16 * 4;
        if (e < p.head_dim) {
          if (whole) *reinterpret_cast<f32x4*>(static_cast<uint8_t*>(p.out) + now.q * p.out_seq + (int64_t)(mm / G) * p.out_row + (int64_t)(now.g * G + mm % G) * p.out_head + e * 4) = y[c] * (1.0f / sum);
          else *reinterpret_cast<f32x4*>(ws.part + ((int64_t)(plan.me * 2 + (now.tile0 == 0 ? 1 : 0)) * BM + r) * (DP + 4) + e) = y[c];
        }
      }
      if (!whole && l16 == 0) {
        float* part = ws.part + ((int64_t)(plan.me * 2 + (now.tile0 == 0 ? 1 : 0)) * BM + r) * (DP + 4);
        part[DP] = top, part[DP + 1] = sum;
      }
    }
    more = plan.following(now);
    if (more) plan.advance(now);
  }
  if (tid == 0) ws.owner[plan.me] = mine;
}

int64_t attention_workspace(int batch, int M, int q_heads, int kv_heads, int head_dim, bool bf16) {
  const AttentionPlan a = plan_attention(M, q_heads, kv_heads, head_dim, bf16);
  return owner_bytes(a.groups) + (int64_t)a.groups * 2 * a.bm * (a.dp + 4) * 4;
}

template <bool BF16, int DP, int MQ, int WK>
static hipError_t launch_attention_t(const AttentionJob& job, const AttentionPlan& plan, hipStream_t st) {
  typedef AttentionShape<BF16, DP, MQ, WK> S;
  const AttentionSpace ws = space_of(job, plan);
  const size_t smem = S::LDS + 2 * (((size_t)job.M + 8) & ~(size_t)7) * sizeof(uint16_t);
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  static std::atomic<uint64_t> allowed{0};   // devices where this kernel may have so much memory, per instantiation
  if (device >= 64 || !((allowed.load(std::memory_order_relaxed) >> device) & 1)) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(attention_kernel<BF16, DP, MQ, WK>), hipFuncAttributeMaxDynamicSharedMemorySize,
                            S::LDS + 2 * ((kMaxTreeItems + 8) & ~7) * (int)sizeof(uint16_t));
    if (e != hipSuccess) return e;
    if (device < 64) allowed.fetch_or(1ull << device, std::memory_order_relaxed);
  }
  hipLaunchKernelGGL((attention_kernel<BF16, DP, MQ, WK>), dim3(plan.groups), dim3(256), smem, st, job, ws);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attention_join_kernel<BF16, DP, S::BM>), dim3(plan.groups, (S::BM + join_rows(DP) - 1) / join_rows(DP)), dim3(256), 0, st, job, ws);
  return hipGetLastError();
}

hipError_t launch_attention(const AttentionJob& job, bool bf16, hipStream_t st) {
  const AttentionPlan a = plan_attention(job.M, job.q_heads, job.kv_heads, job.head_dim, bf16);
  if (!bf16 && a.dp == 256) {
    const AttentionSpace ws = space_of(job, a);
    hipLaunchKernelGGL(attention_wide_kernel, dim3(a.groups), dim3(256), 0, st, job, ws);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((attention_join_kernel<false, 256, kWideRows>), dim3(a.groups, kWideRows / join_rows(256)), dim3(256), 0, st, job, ws);
    return hipGetLastError();
  }
#define LAUNCH(BF16, DP, BM, MQ, WK) \
  if (bf16 == BF16 && a.dp == DP && a.bm == BM) return launch_attention_t<BF16, DP, MQ, WK>(job, a, st)
  LAUNCH(true, 64, 16, 1, 4);
  LAUNCH(true, 64, 32, 1, 2);
  LAUNCH(true, 64, 64, 1, 1);
  LAUNCH(true, 64, 128, 2, 1);
  LAUNCH(true, 128, 16, 1, 4);
  LAUNCH(true, 128, 32, 1, 2);
  LAUNCH(true, 128, 64, 1, 1);
  LAUNCH(true, 128, 128, 2, 1);
  LAUNCH(true, 256, 16, 1, 4);
  LAUNCH(true, 256, 32, 1, 2);
  LAUNCH(true, 256, 64, 1, 1);
  LAUNCH(false, 64, 16, 1, 4);
  LAUNCH(false, 64, 32, 1, 2);
  LAUNCH(false, 64, 64, 1, 1);
  LAUNCH(false, 128, 16, 1, 4);
  LAUNCH(false, 128, 32, 1, 2);
  LAUNCH(false, 128, 64, 1, 1);
#undef LAUNCH
  return hipErrorInvalidValue;
}

}  // namespace specdraft
