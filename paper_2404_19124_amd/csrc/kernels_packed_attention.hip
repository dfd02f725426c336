// Attention of a token tree's rows over a paged cache of four bits and their own ancestors.  The mathematics, the shares, the softmax and
// the products are those of the attention over a cache of 16 bits (attention_body.h); a tile's codes pass through registers on their way
// into LDS, where they lie as the bfloat16 values that they stand for: every value is one, so nothing is rounded.  With many query rows the
// products bound it: 32 sequences of 8 key/value heads with 520 rows each, 225 us, 570 TFLOP/s (a cache of 16
// bits, whose tiles are worked on in the same way: 248).  With few rows it is the reading: see the second kernel.
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

  // item j of a lane (16 lanes write a word each of 16 keys, in banks of their own; a key's groups by neighbours: 226.7 -> 225.7 us)
  static __device__ __forceinline__ int item(int j) { return j * 64 + (threadIdx.x & 63); }
  static __device__ __forceinline__ bool value(int j) { return DP == 64 ? (threadIdx.x & 32) != 0 : j * 64 >= RW * G; }
  static __device__ __forceinline__ int key(int j) { return item(j) % RW; }
  static __device__ __forceinline__ int group(int j) { return item(j) % (RW * G) / RW; }

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

// ---- few query rows: every wave goes through tiles of its own -----------------------------------------------------------------
// A unit of up to 16 query rows has so little work for a key that a workgroup's barriers, not the bytes, would set the pace: here the
// tiles of a segment go round the four waves, which meet at its end only.  Keys go from codes to the operand of the first product in
// registers: lane l16 of group grp holds elements grp * DP/4 on of key l16 of a block of 16, and the queries lie in that order too.
// Values pass through memory of the wave's own, 32 keys at a time, to be read transposed.  A wave's next tile is on its way while it works
// on one; every read of a tile of cached tokens is unconditional, so that none waits for those before it.  64 sequences
// of up to 8000 tokens, 8 heads of 128, one token with 64 heads each, 308 MB, 80 us, 3.9 TB/s, the tiles of
// all four waves in turn by barriers 137 us.  Half of the waves' time is waiting, vector instructions take 32 % of the SIMDs':
// it is not the memory's rate that bounds it (the same call over 16 bits reads 5.0 TB/s).  Every second load fetches one byte of scale to a lane.
// Less work: 32 heads, one sequence of 500 tokens 14.7 -> 12.4 us, 32 of 500, 8 heads 24.2 -> 20.8.
// Two workgroups to a CU: three of 168 registers 91 us.  A page that is no multiple of 16 tokens keeps the barriers: pages of 50 in the call above 157 us.
// Where the heads of a token lie beside each other in a block, not the tokens of a head, so that a head's rows of 64 bytes are apart, it takes 122 us.
constexpr int kStreamRows = 16, kStreamCost = 12;
// (the cost: what a unit's start and end take, in tiles.  The call above, where one sequence has nothing cached, with costs of 2, 6, 12 and 20:
// 103, 88, 80 and 81 us; 8 such sequences 46, 29, 24 and 26; one of 30,000 tokens 30, 30, 30 and 29; 17 rows of 40 heads, 6 sequences 119, 67, 54 and 55; 32
// rows of 8 heads, 16 sequences 55, 34, 31 and 32)
typedef __attribute__((address_space(1))) uint8_t global_u8;
template <int DP>
struct PackedStream {
  typedef AttentionTile<true, DP, 1, 1> Tile;           // (its queries in another order)
  static constexpr int NC = DP / 32, NS = DP > 128 ? 2 : 1;      // words of codes of a lane's quarter of a key, and scales
  static constexpr int NB = KT / 16, ROWB = DP * 2, SWZ = ROWB / 16 < 16 ? ROWB / 16 - 1 : 15;
  static constexpr int PER = DP / 4 + 2;                         // results of a lane
  static constexpr int WAVE = PER * 256, LDS = 4 * WAVE;         // memory of a wave: its values, or its results
  static_assert(32 * ROWB <= WAVE, "values of 32 keys");
  const AttentionJob& p;
  int64_t to_v_rows;
  int last_word;                                        // of a row of bfloat16
  uint64_t k, v, k_scale, v_scale;                      // of the segment's head (what is the same in every lane is in scalar registers)
  uint32_t offset[NS], scale_offset[NS];                // this lane's quarter of key l16 from a block's first key
  uint32_t shift[NS];                                   // of its scale into a float's exponent; behind the head's elements away from it

  // The blocks of 16 keys of 16 tiles from tile `base` on, one to a lane (pages hold whole ones): where they lie, and which of their
  // keys are cached tokens.  What is none is read from the cache's first block, so that no read waits for a decision.
  struct Places {
    int64_t codes, scales;
    int base;
    uint32_t cached;
  };
  struct Codes {                                        // a tile's keys, or its values
    uint32_t c[NB][NC];
    uint32_t scale[NB][NS];
  };

  __device__ __forceinline__ void init() {
    const int lane = threadIdx.x & 63, l16 = lane & 15, grp = lane >> 4;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int e = grp * (DP / 4) + i * 32;
      const bool ok = e < p.head_dim;
      shift[i] = ok ? 23 : 31;   // (there the queries are zeros: any number will do, but for one that is not finite)
      offset[i] = (uint32_t)(l16 * (int)p.slot + (ok ? e / 2 : 0));
      scale_offset[i] = (uint32_t)(l16 * (int)p.scale_slot + (ok ? e / 32 : 0));
    }
  }
  __device__ __forceinline__ void of(const Segment& s) {
    k = uniform(reinterpret_cast<uint64_t>(s.k_cache));
    v = k + (reinterpret_cast<uint64_t>(p.v) - reinterpret_cast<uint64_t>(p.k));
    k_scale = uniform(reinterpret_cast<uint64_t>(p.k_scale + s.g * p.scale_head));
    v_scale = k_scale + (reinterpret_cast<uint64_t>(p.v_scale) - reinterpret_cast<uint64_t>(p.k_scale));
  }
  __device__ __forceinline__ Places places(const Segment& s, int base) const {
    const int key = (s.tile0 + base) * KT + (int)(threadIdx.x & 63) * 16;
    Places r = {0, 0, base, 0};
    if (key < s.ctx) {
      const int b = key / p.block_size, x = p.block_table[(int64_t)s.q * p.max_blocks + b];
      if (x >= 0 && x < p.n_blocks) {
        const int slot = key - b * p.block_size;
        r.codes = x * p.block + slot * p.slot, r.scales = x * p.scale_block + slot * p.scale_slot;
        r.cached = (1u << min(s.ctx - key, 16)) - 1;
      }
    }
    return r;
  }
  static __device__ __forceinline__ uint64_t of_lane(int64_t x, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, lane);
  }
  // Requests tile t's keys, or its values; which of its keys are cached tokens.
  __device__ __forceinline__ uint64_t load(int t, const Places& f, bool value, Codes& x) const {
    uint64_t cached = 0;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int from = (t - f.base) * NB + nb;
      cached |= (uint64_t)(uint32_t)__builtin_amdgcn_readlane(f.cached, from) << nb * 16;
      const global_u8* at = reinterpret_cast<const global_u8*>((value ? v : k) + of_lane(f.codes, from));
      const global_u8* of = reinterpret_cast<const global_u8*>((value ? v_scale : k_scale) + of_lane(f.scales, from));
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        if constexpr (NC == 2) {
          const uint64_t w = *reinterpret_cast<const __attribute__((address_space(1))) uint64_t*>(at + offset[i]);
          x.c[nb][0] = (uint32_t)w, x.c[nb][1] = (uint32_t)(w >> 32);
        } else {
          const u32x4 w = *reinterpret_cast<const __attribute__((address_space(1))) u32x4*>(at + offset[i]);
#pragma unroll
          for (int k = 0; k < 4; ++k) x.c[nb][i * 4 + k] = w[k];
        }
        x.scale[nb][i] = of[scale_offset[i]];
      }
    }
    return cached;
  }
  // Block nb of a tile as bfloat16, this lane's quarter of key l16.  ROWS: some of the tile's keys are not cached tokens but rows of the
  // tree, or none (then row 0)
  template <bool ROWS>
  __device__ __forceinline__ void expand(const Segment& s, int t, const Codes& x, int nb, uint64_t cached, bool value, bool careful, u32x4 (&w)[NC]) const {
#pragma unroll
    for (int i = 0; i < NC; ++i) w[i] = unpack_scaled(x.c[nb][i], __uint_as_float(x.scale[nb][i * NS / NC] << shift[i * NS / NC]));
    if constexpr (ROWS) {
      const int lane = threadIdx.x & 63, l16 = lane & 15, grp = lane >> 4;
      if (!((cached >> (nb * 16 + l16)) & 1)) {
        const int key = (s.tile0 + t) * KT + nb * 16 + l16, row = key >= s.ctx && key < s.keys ? key - s.ctx : 0;
        const uint8_t* from = s.k_rows + row * p.new_row + (value ? to_v_rows : 0) + grp * (DP / 4) * 2;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
          w[i] = (u32x4){0, 0, 0, 0};
          if (grp * (DP / 4) / 8 + i > last_word) continue;
          w[i] = *reinterpret_cast<const u32x4*>(from + i * 16);
          if (careful && value) {   // (see clean_tile)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if ((w[i][j] & 0x7f800000u) == 0x7f800000u) w[i][j] &= 0xffffu;
              if ((w[i][j] & 0x7f80u) == 0x7f80u) w[i][j] &= 0xffff0000u;
            }
          }
        }
      }
    }
  }
};

template <int DP>
__global__ __launch_bounds__(256, DP <= 128 ? 2 : 1) void packed_stream_kernel(AttentionJob p, AttentionSpace ws) {
  typedef PackedStream<DP> Stream;
  typedef typename Stream::Tile Tile;
  constexpr int BM = kStreamRows, NB = Stream::NB, NC = Stream::NC, ND = DP / 16, ROWB = Stream::ROWB;
  extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
  __shared__ int s_odd[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), l16 = lane & 15, grp = lane >> 4;
  const int G = p.q_heads / p.kv_heads;
  Schedule<BM, kStreamCost> plan = {p, G};
  if (!plan.live(ws)) return;
  Segment now;
  Owner mine = {-1, 0, 0, 0, 0};
  bool more = plan.first(now);
  if (!more) {
    if (tid == 0) ws.owner[plan.me] = mine;
    return;
  }
  const int me = plan.me;
  const float q_sign = p.scale < 0 ? -1.0f : p.scale == 0 ? 0.0f : 1.0f;
  const float sc = (p.scale == 0 ? 1.0f : fabsf(p.scale)) * kLog2e;
  Stream in = {p, static_cast<const uint8_t*>(p.v_new) - static_cast<const uint8_t*>(p.k_new), p.head_dim / 8 - 1};
  in.init();
  uint16_t* s_up = reinterpret_cast<uint16_t*>(smem + Stream::LDS);
  lds_u8* vb = (lds_u8*)smem + wave * Stream::WAVE;
  bool careful = false;        // the second pass over this share
  int n_units = 0, first_odd = 1 << 30, unit0 = 0;   // as in attention_body (of all waves: they have the same rows)
  while (more) {
    const int rows = (now.nodes + 1) * G - now.block * BM;
    const bool holds_rows = (now.tile0 + now.n_tiles) * KT > now.ctx;
    const int n_up = holds_rows ? now.keys - now.ctx - 1 : 0;
    int up = tid < n_up ? p.node_parent[(int64_t)now.q * p.M + tid] : 0;   // (on its way with the queries and the places)
    Tile x;
    const int mm = l16 < rows ? now.block * BM + l16 : 0;
    x.row_of[0] = mm / G;
    const uint8_t* from = static_cast<const uint8_t*>(p.q) + now.q * p.q_seq + (int64_t)x.row_of[0] * p.q_row + (int64_t)(now.g * G + mm % G) * p.q_head;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int word = grp * NC + i;
      u32x4 raw = {0, 0, 0, 0};
      if (word <= in.last_word) raw = *reinterpret_cast<const u32x4*>(from + word * 16);
      if (q_sign != 1.0f) {
#pragma unroll
        for (int j = 0; j < 4; ++j) raw[j] = q_sign == 0.0f ? 0u : raw[j] ^ 0x80008000u;
      }
      x.qf[0][i] = __builtin_bit_cast(bf16x8, raw);
    }
    float m_run = kLowest, l_run = 0;
#pragma unroll
    for (int d = 0; d < ND; ++d) x.o[0][d] = (f32x4){0, 0, 0, 0};
    in.of(now);
    const int n_tiles = uniform(now.n_tiles);
    typename Stream::Places f = in.places(now, 0);
    for (int i = tid; i < n_up; i += 256) {
      s_up[i + 1] = (uint16_t)(up >= 0 && up < i ? up + 1 : 0);
      if (i + 256 < n_up) up = p.node_parent[(int64_t)now.q * p.M + i + 256];
    }
    typename Stream::Codes kc, vc;
    uint64_t cached = 0;
    bool odd = false;
    __syncthreads();   // parents are there; the last segment's results have been read
    auto tile = [&](auto has_rows, int t) {
      constexpr bool ROWS = decltype(has_rows)::value;
      const int t0 = (now.tile0 + t) * KT, ctx = now.ctx;
      const uint64_t here = cached;
      // ---- scores, transposed: keys 4 grp + i of a block in the lane's registers, query row l16 ----
      f32x4 s[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        u32x4 kf[NC];
        in.template expand<ROWS>(now, t, kc, nb, here, false, careful, kf);
        s[nb] = (f32x4){0, 0, 0, 0};
#pragma unroll
        for (int st = 0; st < NC; ++st) s[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[st]), x.qf[0][st], s[nb], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      const int next = t + 4 < n_tiles ? t + 4 : t;   // (behind its last tile a wave requests that again: no decision)
      if constexpr (!ROWS) {
        if (next - f.base >= 16) f = in.places(now, next);
        cached = in.load(next, f, false, kc);
        __builtin_amdgcn_sched_barrier(0);
      } else {
        uint64_t sees = here;
        int row = x.row_of[0];
        auto see = [&](int r) {
          const uint32_t bit = (uint32_t)(ctx + r - t0);
          if (bit < (uint32_t)KT) sees |= 1ull << bit;
        };
        if (t0 + KT > ctx) {
          for (int i = 0; i < kMaxStages && row > 0; ++i) {
            see(row);
            row = s_up[row];
          }
          see(0);
        }
        sees >>= grp * 4;
        const uint32_t word[2] = {(uint32_t)sees, (uint32_t)(sees >> 32)};
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!((word[nb / 2] >> ((nb & 1) * 16 + i)) & 1)) s[nb][i] = SPEC_NEG_INF;
      }
      // ---- softmax: weights relative to a bound of the scores ----
      float top = s[0][0];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[nb][i]);
      top = groups_max(top) * sc;
      if (__any(top > m_run)) {
        const float m_new = fmaxf(m_run, top + kSlack), keep = __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
        l_run *= keep;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) x.o[0][d][i] *= keep;
      }
      bf16x8 w[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 raw;
#pragma unroll
        for (int nb = 0; nb < 2; ++nb) {
          float e[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * h + nb][i], sc, -m_run));
          raw[2 * nb] = f32_to_bf16_pair(e[0], e[1]), raw[2 * nb + 1] = f32_to_bf16_pair(e[2], e[3]);
        }
        // (the sum is that of the weights as they are multiplied)
        const bf16x2 one = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t pair = raw[i];   // (of its own: a bit_cast of a vector's element takes the first one)
          l_run = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), one, l_run, false);
        }
        w[h] = __builtin_bit_cast(bf16x8, raw);
      }
      // ---- values, 32 keys at a time (a wave's reads and writes of LDS keep their order) ----
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int nb = 0; nb < 2; ++nb) {
          u32x4 vf[NC];
          in.template expand<ROWS>(now, t, vc, 2 * h + nb, here, true, careful, vf);
          const int key = nb * 16 + l16;
#pragma unroll
          for (int i = 0; i < NC; ++i) *reinterpret_cast<lds_u32x4*>(vb + key * ROWB + (((grp * NC + i) ^ (key & Stream::SWZ)) * 16)) = vf[i];
          __builtin_amdgcn_sched_barrier(0);
        }
        if (h == 1 && !ROWS) in.load(next, f, true, vc);
        __builtin_amdgcn_sched_barrier(0);
        i16x4 v[3][2];   // (two steps' reads are under way)
        auto read = [&](int d) {
#pragma unroll
          for (int nb = 0; nb < 2; ++nb) {
            const int key = nb * 16 + grp * 4 + (l16 >> 2), word = (d * 2 + ((l16 & 3) >> 1)) ^ (key & Stream::SWZ);
            v[d % 3][nb] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vb + key * ROWB + word * 16 + (l16 & 1) * 8));
          }
        };
        read(0);
        read(1);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          if (d + 2 < ND) read(d + 2);
          __builtin_amdgcn_sched_barrier(0);
          const i16x4 a = v[d % 3][0], b = v[d % 3][1];
          x.o[0][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, (i16x8){a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}), w[h], x.o[0][d], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    };
    // tiles of cached tokens, each requested while the one before is worked on; the others, a share's last ones, when it is their turn
#pragma unroll 1
    for (int t = wave; t < n_tiles; t += 4) {
      if (t - f.base >= 16) f = in.places(now, t);
      cached = in.load(t, f, false, kc);
      __builtin_amdgcn_sched_barrier(0);
      in.load(t, f, true, vc);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll 1
      for (; cached == ~0ull && t < n_tiles; t += 4) tile(std::false_type(), t);
      if (t >= n_tiles) break;
      odd = true;
      tile(std::true_type(), t);
    }
    l_run = groups_sum(l_run);

    // ---- join of the waves: each one joins a quarter of the head ----
    auto mine_is = [&](int d) { return d / (ND / 4) == wave; };
    float* box = reinterpret_cast<float*>(smem) + lane;
    constexpr int PER = Stream::PER;
    box[wave * PER * 64] = m_run;
    box[(wave * PER + 1) * 64] = l_run;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) box[(wave * PER + 2 + d * 4 + i) * 64] = x.o[0][d][i];
    if (lane == 0) s_odd[wave] = odd;
    __syncthreads();
    float part[4];
    m_run = kLowest, l_run = 0;
#pragma unroll
    for (int y = 0; y < 4; ++y) part[y] = box[y * PER * 64], m_run = fmaxf(m_run, part[y]);
#pragma unroll
    for (int y = 0; y < 4; ++y) part[y] = __builtin_amdgcn_exp2f(part[y] - m_run), l_run = __builtin_fmaf(box[(y * PER + 1) * 64], part[y], l_run);
    bool finite = true;
#pragma unroll
    for (int d = 0; d < ND; ++d)
      if (mine_is(d)) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float o = 0;
#pragma unroll
          for (int y = 0; y < 4; ++y) o = __builtin_fmaf(box[(y * PER + 2 + d * 4 + i) * 64], part[y], o);
          x.o[0][d][i] = o;
          finite = finite && o * 0.0f == 0.0f;
        }
      }
    const bool whole = now.n_seg == now.tiles;
    if (!whole && now.tile0 == 0) mine = {now.q, now.g, now.block, plan.last(), min(rows, BM)};
    if (!careful && (s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3]) && __syncthreads_or(!finite)) first_odd = min(first_odd, n_units);
    if (careful && holds_rows)
      add_left_out(x, now.k_rows, in.to_v_rows, p.new_row, now.ctx, now.tile0 * KT, (now.tile0 + now.n_tiles) * KT, s_up, in.last_word);
    if (l16 < rows && (careful ? n_units - unit0 >= first_odd : n_units < first_odd)) {
      const float inv = whole ? 1.0f / l_run : 1.0f;
      uint8_t* out = static_cast<uint8_t*>(p.out) + now.q * p.out_seq + (int64_t)x.row_of[0] * p.out_row + (int64_t)(now.g * G + mm % G) * p.out_head;
      float* to = ws.part + ((int64_t)(me * 2 + (now.tile0 == 0 ? 1 : 0)) * BM + l16) * (DP + 4);
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const int e = d * 16 + grp * 4;
        if (!mine_is(d)) continue;
        const f32x4 v = x.o[0][d] * inv;
        if (!whole) *reinterpret_cast<f32x4*>(to + e) = v;
        else if (e < p.head_dim) *reinterpret_cast<uint64_t*>(out + e * 2) = (uint64_t)f32_to_bf16_pair(v[2], v[3]) << 32 | f32_to_bf16_pair(v[0], v[1]);
      }
      if (!whole && wave == 0 && grp == 0) to[DP] = m_run, to[DP + 1] = l_run;
    }
    more = plan.following(now);
    if (more) plan.advance(now);
    ++n_units;
    if (careful) __syncthreads();   // the parents have been read
    if (!more && !careful && first_odd < n_units) {
      careful = true;
      unit0 = n_units;
      more = plan.first(now);
    }
  }
  if (tid == 0) ws.owner[me] = mine;
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

template <int DP>
static hipError_t launch_stream_t(const AttentionJob& job, const AttentionPlan& plan, hipStream_t st) {
  const AttentionSpace ws = space_of(job, plan);
  const size_t smem = PackedStream<DP>::LDS + (((size_t)job.M + 8) & ~(size_t)7) * sizeof(uint16_t);
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  static std::atomic<uint64_t> allowed{0};   // devices where this kernel may have so much memory, per instantiation
  if (device >= 64 || !((allowed.load(std::memory_order_relaxed) >> device) & 1)) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(packed_stream_kernel<DP>), hipFuncAttributeMaxDynamicSharedMemorySize,
                            PackedStream<DP>::LDS + ((kMaxTreeItems + 8) & ~7) * (int)sizeof(uint16_t));
    if (e != hipSuccess) return e;
    if (device < 64) allowed.fetch_or(1ull << device, std::memory_order_relaxed);
  }
  hipLaunchKernelGGL((packed_stream_kernel<DP>), dim3(plan.groups), dim3(256), smem, st, job, ws);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((attention_join_kernel<true, DP, kStreamRows>), dim3(plan.groups, (kStreamRows + join_rows(DP) - 1) / join_rows(DP)), dim3(256), 0, st, job, ws);
  return hipGetLastError();
}

// The streams' plan (no more workspace than the other's); bm 0: too many query rows for a key/value head.  More than 16 of them are two units, which read the same keys beside each
// other: 17 rows of 40 heads, 6 sequences of up to 9600 tokens 92 -> 54 us (their bytes at a sum's rate: 43), 32 rows of 8 heads, 16 of up to 4000 44 -> 31 (10);
// but three and four
// units 42 -> 46 us (48 rows, 8 heads, 32 of 2000) and 73 -> 83 (49 rows, 32 heads, 16 of 2000).
static AttentionPlan plan_streams(int M, int q_heads, int kv_heads, int head_dim) {
  AttentionPlan a = plan_attention(M, q_heads, kv_heads, head_dim, true);
  a.bm = a.bm <= 2 * kStreamRows ? kStreamRows : 0;
  a.least = 4;
  return a;
}

hipError_t launch_packed_attention(const AttentionJob& job, hipStream_t st) {
  const AttentionPlan few = plan_streams(job.M, job.q_heads, job.kv_heads, job.head_dim);
  if (few.bm && job.one_place)
    return few.dp == 64 ? launch_stream_t<64>(job, few, st) : few.dp == 128 ? launch_stream_t<128>(job, few, st) : launch_stream_t<256>(job, few, st);
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
