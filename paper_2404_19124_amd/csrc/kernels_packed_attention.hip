// Attention of a token tree's rows over a paged cache of four bits and their own ancestors.  The mathematics, the shares, the softmax and
// the products are those of the attention over a cache of 16 bits (attention_body.h); a tile's codes pass through registers on their way
// into LDS, where they lie as the bfloat16 values that they stand for: every value is one, so nothing is rounded.
#include <atomic>

#include "attention_body.h"
#include "packed.h"

namespace specdraft {

// How a workgroup brings tiles into LDS.  A wave takes 16 of a tile's 64 keys, a lane NI groups of 32 elements, 16 bytes of codes and a
// scale each: they are requested two tiles ahead, and written as bfloat16 one tile ahead, when the other buffer is free.  Rows of the
// tree are copied straight into LDS, as everything is in the attention over 16 bits.  Where the wave's 16 tokens lie in one page their
// place is one address for all lanes, found for 64 tiles at once, a tile per lane.
template <int DP, int MQ, int WK>
struct PackedCopy {
  typedef AttentionShape<true, DP, MQ, WK> S;
  static constexpr bool kEarly = true;
  static constexpr int RW = KT / 4, G = DP / 32, NI = G / 2;   // keys of a wave, groups of a key, groups of a lane
  static constexpr int RPI = 64 / S::CH, NL = RW / RPI;        // rows and number of the instructions that copy tree rows
  const AttentionJob& p;
  uint32_t (*s_valid)[4];
  int last_word;
  int64_t to_v_cache, to_v_rows;               // from a key to its value
  uint32_t offset[NI], scale_offset[NI];       // of this lane's groups from the place of the wave's rows
  bool pending;                                // copies of tree rows are on their way

  struct Places {
    int block, slot;   // of the wave's rows of 64 tiles from tile `base` on (lane by lane, block -1: no single place)
    int base;
  };
  struct Source {
    uint64_t k_cache, k_rows;   // 0: nothing to copy
    uint32_t valid;             // which of the wave's rows are cached tokens
    int row;                    // lane l: the tree's row that is row l % 16 (where not all of them are)
    u32x4 code[NI];
    uint32_t scale[NI];
  };
  static __device__ __forceinline__ Source nothing() { return {0, 0, 0, 0, {}, {}}; }

  // item j of a lane
  static __device__ __forceinline__ int item(int j) { return j * 64 + (threadIdx.x & 63); }
  static __device__ __forceinline__ bool value(int j) { return DP == 64 ? (threadIdx.x & 32) != 0 : j * 64 >= RW * G; }
  static __device__ __forceinline__ int key(int j) { return item(j) % (RW * G) / G; }
  static __device__ __forceinline__ int group(int j) { return item(j) % G; }

  __device__ __forceinline__ void landed() {
    if (pending) __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));   // vmcnt(0)
    pending = false;
  }

  __device__ __forceinline__ void init() {
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      offset[j] = (uint32_t)(key(j) * (int)p.slot + group(j) * 16);
      scale_offset[j] = (uint32_t)(key(j) * (int)p.scale_slot + group(j));
    }
    pending = false;
  }

  __device__ __forceinline__ Places places(const Segment& s, int base) const {
    const int lane = threadIdx.x & 63, key = (s.tile0 + base + lane) * KT + (int)(threadIdx.x >> 6) * RW;
    Places r = {-1, 0, base};
    if (p.one_place && key + RW <= s.ctx && base + lane < s.n_tiles) {
      const int b = key / p.block_size, x = p.block_table[(int64_t)s.q * p.max_blocks + b];
      if (x >= 0 && x < p.n_blocks) r.block = x, r.slot = key - b * p.block_size;
    }
    return r;
  }
  __device__ __forceinline__ Source source(const Segment& s, int t, Places& f) const {
    if (t - f.base == 64) f = places(s, t);
    Source x = nothing();
    x.k_cache = reinterpret_cast<uint64_t>(s.k_cache), x.k_rows = reinterpret_cast<uint64_t>(s.k_rows);
    const int block = __builtin_amdgcn_readlane(f.block, t - f.base);
    const uint8_t *k_scale = p.k_scale + s.g * p.scale_head, *v_scale = p.v_scale + s.g * p.scale_head;
    if (block >= 0) {
      const int slot = __builtin_amdgcn_readlane(f.slot, t - f.base);
      const int64_t place = block * p.block + slot * p.slot, scale_place = block * p.scale_block + slot * p.scale_slot;
      x.valid = (1u << RW) - 1;
#pragma unroll
      for (int j = 0; j < NI; ++j) {
        if (group(j) * 4 > last_word) continue;
        x.code[j] = *reinterpret_cast<const u32x4*>(s.k_cache + place + (value(j) ? to_v_cache : 0) + offset[j]);
        x.scale[j] = ((value(j) ? v_scale : k_scale) + scale_place)[scale_offset[j]];
      }
      return x;
    }
    // what is not a key is read from row 0, which every row sees: with a weight of zero it adds nothing
    const int tid = opaque_tid(), key0 = (s.tile0 + t) * KT + (tid >> 6) * RW + (tid & 63) % RW;
    int y = -1, slot = 0;
    if (key0 < s.ctx) {
      const int b = key0 / p.block_size;
      y = p.block_table[(int64_t)s.q * p.max_blocks + b];
      slot = key0 - b * p.block_size;
    } else if (key0 < s.keys) {
      x.row = key0 - s.ctx;
    }
    x.valid = (uint32_t)__ballot(y >= 0 && y < p.n_blocks) & ((1u << RW) - 1);
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int64_t b = __shfl(y, key(j)), in = __shfl(slot, key(j));
      if (!((x.valid >> key(j)) & 1) || group(j) * 4 > last_word) continue;
      x.code[j] = *reinterpret_cast<const u32x4*>(s.k_cache + b * p.block + in * p.slot + (value(j) ? to_v_cache : 0) + group(j) * 16);
      x.scale[j] = ((value(j) ? v_scale : k_scale) + b * p.scale_block + in * p.scale_slot)[group(j)];
    }
    return x;
  }

  __device__ __forceinline__ static void copy16(uint64_t from, uint32_t offset, lds_u8* to) {
    const auto place = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(uniform(from)), 0, -1, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(place, (__attribute__((address_space(3))) void*)to, 16, offset, 0, 0, 0);
  }

  __device__ __forceinline__ void copy(const Source& s, lds_u8* to, uint32_t* valid) {
    const int tid = opaque_tid(), lane = tid & 63, wave = uniform(tid >> 6);
    if (lane == 0) valid[wave] = s.valid;
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      if (!((s.valid >> key(j)) & 1)) continue;
      const int row = wave * RW + key(j);
      const uint32_t base = row * S::ROWB + ((group(j) * 4) ^ (row & S::SWZ)) * 16 + (value(j) ? KT * S::ROWB : 0);
#pragma unroll
      for (int w = 0; w < 4; ++w) *reinterpret_cast<lds_u32x4*>(to + (base ^ (w * 16))) = unpack_word(s.code[j][w], s.scale[j]);
    }
    if (s.valid == (1u << RW) - 1) return;
    // ---- rows of the tree: a lane's 16 bytes land at its place in the instruction's 1 KiB ----
    pending = true;
    lds_u8* at = to + wave * RW * S::ROWB;
    if (p.offsets_fit) {
#pragma unroll
      for (int j = 0; j < NL; ++j) {
        const int row = j * RPI + lane / S::CH, word = min((lane % S::CH) ^ ((wave * RW + row) & S::SWZ), last_word);
        const uint32_t from = (uint32_t)__shfl(s.row, row) * (uint32_t)p.new_row + word * 16;
        if (!((s.valid >> row) & 1)) {
          copy16(s.k_rows, from, at + j * RPI * S::ROWB);
          copy16(s.k_rows + to_v_rows, from, at + (KT + j * RPI) * S::ROWB);
        }
      }
      return;
    }
#pragma unroll 1
    for (int row = 0; row < RW; ++row) {   // (rows more than 4 GiB apart) row by row, by the lanes whose words are theirs
      const uint64_t k = s.k_rows + (uint64_t)(__builtin_amdgcn_readlane(s.row, row) * p.new_row);
      const int word = (lane % S::CH) ^ ((wave * RW + row) & S::SWZ), j = row / RPI;
      if (!((s.valid >> row) & 1) && lane / S::CH == row % RPI) {
        copy16(k, min(word, last_word) * 16, at + j * RPI * S::ROWB);
        copy16(k + to_v_rows, min(word, last_word) * 16, at + (KT + j * RPI) * S::ROWB);
      }
    }
  }
};

template <int DP, int MQ, int WK>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void packed_attention_kernel(AttentionJob p, AttentionSpace ws) {
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  __shared__ uint32_t s_valid[2][4], s_again;
  attention_body<true, DP, MQ, WK, PackedCopy<DP, MQ, WK>>(p, ws, smem, s_valid, s_again);
}

template <int DP, int MQ, int WK>
static hipError_t launch_packed_t(const AttentionJob& job, const AttentionPlan& plan, hipStream_t st) {
  typedef AttentionShape<true, DP, MQ, WK> S;
  const AttentionSpace ws = space_of(job, plan);
  const size_t smem = S::LDS + 2 * (((size_t)job.M + 8) & ~(size_t)7) * sizeof(uint16_t);
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  static std::atomic<uint64_t> allowed{0};   // devices where this kernel may have so much memory, per instantiation
  if (device >= 64 || !((allowed.load(std::memory_order_relaxed) >> device) & 1)) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(packed_attention_kernel<DP, MQ, WK>), hipFuncAttributeMaxDynamicSharedMemorySize,
                            S::LDS + 2 * ((kMaxTreeItems + 8) & ~7) * (int)sizeof(uint16_t));
    if (e != hipSuccess) return e;
    if (device < 64) allowed.fetch_or(1ull << device, std::memory_order_relaxed);
  }
  hipLaunchKernelGGL((packed_attention_kernel<DP, MQ, WK>), dim3(plan.groups), dim3(256), smem, st, job, ws);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attention_join_kernel<true, DP, S::BM>), dim3(plan.groups, (S::BM + join_rows(DP) - 1) / join_rows(DP)), dim3(256), 0, st, job, ws);
  return hipGetLastError();
}

hipError_t launch_packed_attention(const AttentionJob& job, hipStream_t st) {
  const AttentionPlan a = plan_attention(job.M, job.q_heads, job.kv_heads, job.head_dim, true);
#define LAUNCH(DP, BM, MQ, WK) \
  if (a.dp == DP && a.bm == BM) return launch_packed_t<DP, MQ, WK>(job, a, st)
  LAUNCH(64, 16, 1, 4);
  LAUNCH(64, 32, 1, 2);
  LAUNCH(64, 64, 1, 1);
  LAUNCH(64, 128, 2, 1);
  LAUNCH(128, 16, 1, 4);
  LAUNCH(128, 32, 1, 2);
  LAUNCH(128, 64, 1, 1);
  LAUNCH(128, 128, 2, 1);
  LAUNCH(256, 16, 1, 4);
  LAUNCH(256, 32, 1, 2);
  LAUNCH(256, 64, 1, 1);
#undef LAUNCH
  return hipErrorInvalidValue;
}

}  // namespace specdraft
