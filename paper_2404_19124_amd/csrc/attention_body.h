// Attention of a token tree's rows over a paged cache and their own ancestors: what its kernels share.  The mathematics, what bounds them
// and what they measure: kernels_tree_attention.hip, and kernels_packed_attention.hip for a cache of four bits.
#pragma once
#include <type_traits>

#include "device_utils.h"
#include "rows_internal.h"
#include "spec_internal.h"

namespace specdraft {


typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) float lds_f32;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int KT = 64;   // keys of a tile
// How far above the largest score so far the bound is set when it has to move (powers of 2): scores that rise by less leave it where
// it is.  No weight is above 1, so that the largest values' products stay finite, and the largest is 2^-8 at least.
constexpr float kSlack = 8;

// larger / sum of a value and those of the lanes 16 and 32 away: the same query row's other keys
__device__ __forceinline__ float groups_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const uint32_t w = __float_as_uint(x);
  const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float groups_sum(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const uint32_t w = __float_as_uint(x);
  const auto b = __builtin_amdgcn_permlane16_swap(w, w, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// values that are the same in every lane, in scalar registers
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// words that nobody writes while the kernel runs, at addresses that are the same in every lane: scalar loads
typedef const __attribute__((address_space(4))) int32_t* scalar_i32;

// The work is cut into equal shares by COST: a unit costs its tiles and kUnitCost more for its queries and results (a sequence
// with nothing cached, 24 units of one tile in one share: that workgroup took a third longer than all others).  32 sequences of
// 8 key/value heads with 360 query rows: 0: 298 us, 1: 240 us, 2: 221 us, 3: 233 us; float32 tiles take longer, and a cost of 1 is best.
constexpr int unit_cost(bool bf16) { return bf16 ? 2 : 1; }

struct SeqTiles {
  int ctx, nodes, tiles, blocks;   // cached tokens, last row, tiles per unit, units per key/value head
  uint64_t total;                  // cost of all units
};
template <bool UNIFORM = false>
__device__ __forceinline__ SeqTiles seq_tiles(const AttentionJob& p, int q, int BM, int unit_cost) {
  SeqTiles s;
  int ctx, nodes;
  if (UNIFORM) {
    ctx = *(scalar_i32)(p.ctx_len + q);
    nodes = p.n_nodes ? *(scalar_i32)(p.n_nodes + q) : p.M;
  } else {
    ctx = p.ctx_len[q];
    nodes = p.n_nodes ? p.n_nodes[q] : p.M;
  }
  s.ctx = min(max(ctx, 0), p.max_blocks * p.block_size);
  s.nodes = min(max(nodes, -1), p.M);
  s.tiles = (s.ctx + s.nodes + KT) / KT;
  s.blocks = (int)(((int64_t)(s.nodes + 1) * (p.q_heads / p.kv_heads) + BM - 1) / BM);
  s.total = (uint64_t)(s.tiles + unit_cost) * (uint64_t)s.blocks * (uint64_t)p.kv_heads;
  return s;
}

// Shares of up to this cost go to one workgroup per CU, more of them to two.  With one and with two, at shares of 12, 16, 20 and 24: three
// sequences of 32 heads of their own 28.1 / 30.9, 34.0 / 35.1, 48.6 / 47.9 and 55.5 / 55.1 us; 12 sequences of 6 rows, one key/value head, 43.3 /
// 46.3, 46.9 / 47.5, 55.7 / 49.8 and 59.4 / 53.6.  Where heads are shared by 8 and there are many rows, two are faster from 12 on (46.4 / 41.8).
constexpr uint64_t kFewCost = 20;

// What a workgroup that ends inside a unit leaves: see the join below.
struct Owner {
  int q, g, block, last;   // the unit that starts in this workgroup and ends in workgroup `last`; q < 0: none
  int rows;                // its query rows
};

struct AttentionSpace {
  int* live;        // workgroups that have a share
  Owner* owner;     // [groups], of those
  float* part;      // [groups][2][BM][DP + 4]: o, m, l of the segment that goes on from an earlier workgroup, of the one that
                    // goes on to a later one
  int groups;       // workgroups of the launch
  int least;        // cost that a workgroup takes at least
};

// two buffers of keys and values
constexpr int tile_bytes(int one) { return 4 * one; }

template <bool BF16, int DP, int MQ, int WK>
struct AttentionShape {
  static constexpr int ESZ = BF16 ? 2 : 4, ROWB = DP * ESZ, CH = ROWB / 16;   // bytes and 16-byte words of a row
  static constexpr int WQ = 4 / WK, BM = 16 * MQ * WQ;                        // waves along the query rows; query rows of a unit
  static constexpr int KW = KT / WK, NB = KW / 16;                            // keys of a wave, blocks of 16 of them
  static constexpr int LDS = tile_bytes(KT * ROWB);
  static constexpr int SWZ = CH < 16 ? CH - 1 : 15;
  // joins of the waves that share query rows go through the memory of one tile
  static_assert((WK - 1) * WQ * 64 * MQ * (DP / 4 + 2) * 4 <= LDS / 2, "the waves' results fit a tile's memory");
};

// One tile of one unit: scores, softmax and values of a wave's keys and query rows.
template <bool BF16, int DP, int MQ, int WK>
struct AttentionTile {
  typedef AttentionShape<BF16, DP, MQ, WK> S;
  typedef typename std::conditional<BF16, bf16x8, f32x4>::type qword;
  static constexpr int QS = BF16 ? DP / 32 : DP / 16;   // steps along the head
  qword qf[MQ][QS];       // queries: lane l16 of every group holds row l16 of each block of 16
  int row_of[MQ];         // tree rows of this lane's query rows
  f32x4 o[MQ][DP / 16];   // transposed: elements 16 d + 4 grp + i of the head, query row l16
  float m_run[MQ], l_run[MQ];

  // `sees_cached`: which of the tile's keys are cached tokens; t0: its first key
  __device__ __forceinline__ void step(const lds_u8* kb, const lds_u8* vb, uint64_t cached, int t0, int ctx, const uint16_t* s_up, float sc) {
    constexpr int ROWB = S::ROWB, KW = S::KW, NB = S::NB, SWZ = S::SWZ;
    const int tid = opaque_tid(), lane = tid & 63, l16 = lane & 15, grp = lane >> 4, wk = (tid >> 6) % WK;
    // ---- scores, transposed: keys 4 grp + i of a block in the lane's registers, query row l16 ----
    // The reads of the next block of keys are sent before the products of one, and nothing is moved across the line between
    // them: the compiler by itself waits for nearly every read right behind it, in registers that it uses for all of them.
    f32x4 s[MQ][NB];
    u32x4 kf[2][QS];
    auto read_keys = [&](int nb) {
      const int key = wk * KW + nb * 16 + l16;
#pragma unroll
      for (int st = 0; st < QS; ++st) kf[nb & 1][st] = *reinterpret_cast<const lds_u32x4*>(kb + key * ROWB + (((st * 4 + grp) ^ (key & SWZ)) * 16));
    };
    read_keys(0);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (nb + 1 < NB) read_keys(nb + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int mq = 0; mq < MQ; ++mq) s[mq][nb] = (f32x4){0, 0, 0, 0};
#pragma unroll
      for (int st = 0; st < QS; ++st) {
        const qword f = __builtin_bit_cast(qword, kf[nb & 1][st]);
#pragma unroll
        for (int mq = 0; mq < MQ; ++mq) {
          if constexpr (BF16) {
            s[mq][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, qf[mq][st], s[mq][nb], 0, 0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[mq][nb] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[e], qf[mq][st][e], s[mq][nb], 0, 0, 0);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }

    // ---- which of the tile's keys a row sees ----
    if (cached != ~0ull) {
#pragma unroll
      for (int mq = 0; mq < MQ; ++mq) {
        uint64_t sees = cached;
        int row = row_of[mq];
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
        sees >>= wk * KW + grp * 4;
        const uint32_t word[2] = {(uint32_t)sees, (uint32_t)(sees >> 32)};
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!((word[nb / 2] >> ((nb & 1) * 16 + i)) & 1)) s[mq][nb][i] = SPEC_NEG_INF;
      }
    }

    // ---- values.  The weights are in the place that the product wants them in if the values' keys are taken in the same
    // order: 4 grp + i of a block, then of the next.  Two blocks of the head's elements are read ahead, the first ones before the
    // exponentials ----
    constexpr int ND = DP / 16, AHEAD = 2;
    i16x4 vf[AHEAD + 1][NB];
    auto read_values = [&](int d) {
      if constexpr (BF16) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const int key = wk * KW + nb * 16 + grp * 4 + (l16 >> 2), word = (d * 2 + ((l16 & 3) >> 1)) ^ (key & SWZ);
          // (16 lanes read four keys' 16 elements, and each gets one element of the four keys)
          vf[d % (AHEAD + 1)][nb] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vb + key * ROWB + word * 16 + (l16 & 1) * 8));
        }
      }
    };

    // ---- softmax: weights relative to a bound of the scores ----
#pragma unroll
    for (int mq = 0; mq < MQ; ++mq) {
      float top = s[mq][0][0];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[mq][nb][i]);
      top = groups_max(top) * sc;
      // (moving it with every larger score: 128 of a tile's 330 vector instructions)
      if (__any(top > m_run[mq])) {
        const float m_new = fmaxf(m_run[mq], top + kSlack), keep = __builtin_amdgcn_exp2f(m_run[mq] - m_new);
        m_run[mq] = m_new;
        l_run[mq] *= keep;
#pragma unroll
        for (int d = 0; d < DP / 16; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[mq][d][i] *= keep;
      }
    }
    if constexpr (BF16) {
#pragma unroll
      for (int d = 0; d < AHEAD; ++d) read_values(d);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int mq = 0; mq < MQ; ++mq) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mq][nb][i], sc, -m_run[mq]));
          s[mq][nb][i] = w;
          if constexpr (!BF16) l_run[mq] += w;
        }
    }
    // The weights are rounded to bfloat16 for their product with the values, since products of float32 run at an eighth of the rate.  That adds to
    // the rounding of the result: off from 64 bits by 1.60e-3 to 1.70e-3 relative, 1.57e-3 to 1.61e-3 with float32 weights.
    // (the sum is that of the weights as they are multiplied: equal values come out as they are, whatever the rounding)
    auto sum = [&](int mq, uint32_t pair) {
      const bf16x2 one = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
      l_run[mq] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), one, l_run[mq], false);
    };

    if constexpr (BF16) {
      if constexpr (NB == 1) {
        i16x4 w[MQ];
#pragma unroll
        for (int mq = 0; mq < MQ; ++mq) {
          const uint32_t lo = f32_to_bf16_pair(s[mq][0][0], s[mq][0][1]), hi = f32_to_bf16_pair(s[mq][0][2], s[mq][0][3]);
          w[mq] = __builtin_bit_cast(i16x4, (uint64_t)hi << 32 | lo);
          sum(mq, lo);
          sum(mq, hi);
        }
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) {
          if (d + AHEAD < ND) read_values(d + AHEAD);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int mq = 0; mq < MQ; ++mq) o[mq][d] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(vf[d % (AHEAD + 1)][0], w[mq], o[mq][d], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        }
      } else {
        bf16x8 w[MQ][NB / 2];
#pragma unroll
        for (int mq = 0; mq < MQ; ++mq)
#pragma unroll
          for (int j = 0; j < NB / 2; ++j) {
            const f32x4 a = s[mq][2 * j], b = s[mq][2 * j + 1];
            const u32x4 raw = {f32_to_bf16_pair(a[0], a[1]), f32_to_bf16_pair(a[2], a[3]), f32_to_bf16_pair(b[0], b[1]), f32_to_bf16_pair(b[2], b[3])};
            w[mq][j] = __builtin_bit_cast(bf16x8, raw);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum(mq, raw[i]);
          }
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          if (d + AHEAD < ND) read_values(d + AHEAD);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int j = 0; j < NB / 2; ++j) {
            const i16x4 a = vf[d % (AHEAD + 1)][2 * j], b = vf[d % (AHEAD + 1)][2 * j + 1];
            const bf16x8 v = __builtin_bit_cast(bf16x8, (i16x8){a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
#pragma unroll
            for (int mq = 0; mq < MQ; ++mq) o[mq][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, w[mq][j], o[mq][d], 0, 0, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    } else {
      float vr[2][ND];
      auto read_key = [&](int x) {
        const int key = wk * KW + (x >> 2) * 16 + grp * 4 + (x & 3);
#pragma unroll
        for (int d = 0; d < ND; ++d)
          vr[x & 1][d] = *reinterpret_cast<const lds_f32*>(vb + key * ROWB + ((d * 4 + (l16 >> 2)) ^ (key & SWZ)) * 16 + (l16 & 3) * 4);
      };
      read_key(0);
#pragma unroll
      for (int x = 0; x < NB * 4; ++x) {
        if (x + 1 < NB * 4) read_key(x + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int mq = 0; mq < MQ; ++mq) o[mq][d] = __builtin_amdgcn_mfma_f32_16x16x4f32(vr[x & 1][d], s[mq][x >> 2][x & 3], o[mq][d], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
};

// What a careful pass has left out of its rows' sums: the values that are not finite of the rows of the tree that each sees, of those
// that are keys of the segment (key ctx + row in [from, to)).  A weight is above zero, and times such a value that value, but where the
// key is not finite: there the sum is NaN, be the weight zero or not a number itself.
template <bool BF16, int DP, int MQ, int WK>
__device__ __forceinline__ void add_left_out(AttentionTile<BF16, DP, MQ, WK>& x, const uint8_t* k_rows, int64_t to_v, int64_t stride, int ctx, int from, int to,
                                             const uint16_t* s_up, int last_word) {
  constexpr int ESZ = BF16 ? 2 : 4;
  const int grp = (opaque_tid() & 63) >> 4;
  auto finite = [](uint32_t bits) { return BF16 ? (bits & 0x7f80) != 0x7f80 && (bits & 0x7f800000) != 0x7f800000 : (bits & 0x7f800000) != 0x7f800000; };
#pragma unroll
  for (int mq = 0; mq < MQ; ++mq) {
    int row = x.row_of[mq];
    bool sees = true;
#pragma unroll 1
    for (int n = 0; n <= kMaxStages; ++n) {
      const bool here = sees && ctx + row >= from && ctx + row < to;
      const uint8_t *k = k_rows + row * stride, *v = k + to_v;
      float w = 1;
#pragma unroll 1
      for (int word = 0; word <= last_word; ++word) {
        const u32x4 raw = *reinterpret_cast<const u32x4*>(k + word * 16);
        if (!finite(raw[0]) || !finite(raw[1]) || !finite(raw[2]) || !finite(raw[3])) w = __builtin_nanf("");
      }
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) {
        const int e = d * 16 + grp * 4;
        if (!here || e * ESZ > last_word * 16 + 15) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float y = BF16 ? bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(v)[e + i]) : reinterpret_cast<const float*>(v)[e + i];
          if (!(y * 0.0f == 0.0f)) x.o[mq][d][i] += w * y;
        }
      }
      sees = sees && row > 0;
      row = row > 0 && n + 1 < kMaxStages ? s_up[row] : 0;
    }
  }
}

// A weight of zero does not take out a value that is not finite, of a row of the tree that only some rows see, and a zero of a query
// not what stands behind the elements of a key (copies of its last 16 bytes).  Where segments with such keys have sums that are
// not finite, the workgroup goes through its share a second time, CAREFULLY: in every tile that has landed, zeros take the place of what
// is behind the elements and of the values that are not finite of all that is not a cached token.  (In every pass over a tile with rows
// of the tree: 41 -> 46 us for 64 sequences of 100 tokens.  Key by key for every row of such a wave: 45 us -> 16 ms with one infinity among
// 16 sequences of up to 3000 tokens; so: 32 of 45 rows over up to 4000 212 -> 443 us.)
template <bool BF16, int DP, int MQ, int WK>
__device__ __forceinline__ void clean_tile(lds_u8* cur, uint64_t cached, int last_word) {
  typedef AttentionShape<BF16, DP, MQ, WK> S;
  constexpr uint32_t kExponent = BF16 ? 0x7f80 : 0x7f800000;
  for (int i = opaque_tid(); i < KT * S::CH; i += 256) {
    const int key = i / S::CH, word = (i % S::CH) ^ (key & S::SWZ);
    if (word > last_word) *reinterpret_cast<lds_u32x4*>(cur + i * 16) = (u32x4){0, 0, 0, 0};
    if ((cached >> key) & 1) continue;
    lds_u32x4* at = reinterpret_cast<lds_u32x4*>(cur + KT * S::ROWB + i * 16);
    u32x4 v = *at;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (BF16 && ((v[j] >> 16) & kExponent) == kExponent) v[j] &= 0xffffu;
      if ((v[j] & kExponent) == kExponent) v[j] = BF16 ? v[j] & 0xffff0000u : 0u;
    }
    *at = v;
  }
}

// One turn of a workgroup: tile `cur` has landed; the next one is copied into `other` while it is worked on, and (by copies that pass
// through registers) the one behind that is requested.  `odd`: there was a key
// that clean_tile would change.
template <bool BF16, int DP, int MQ, int WK, typename Landed, typename Copy, typename Fetch>
__device__ __forceinline__ void attention_turn(AttentionTile<BF16, DP, MQ, WK>& x, lds_u8* __restrict cur, lds_u8* __restrict other, const uint32_t* valid,
                                               int t0, int ctx, const uint16_t* s_up, float sc, bool active, bool careful, int last_word, bool& odd,
                                               Landed&& landed, Copy&& copy_next, Fetch&& fetch) {
  // this wave's copies have landed, and behind the barrier the others'; all are done with the other buffer
  landed();
  __syncthreads();
  copy_next(other);
  fetch();
  uint64_t cached = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) cached |= (uint64_t)valid[w] << (w * (KT / 4));
  odd |= cached != ~0ull;
  if (careful) {
    clean_tile<BF16, DP, MQ, WK>(cur, cached, last_word);
    __syncthreads();
  }
  if (active) x.step(cur, cur + KT * AttentionShape<BF16, DP, MQ, WK>::ROWB, cached, t0, ctx, s_up, sc);
}

// A unit's tiles that a workgroup takes, in scalar registers.
struct Segment {
  int q, g, block;                   // sequence, key/value head, block of BM query rows
  int ctx, nodes, tiles, blocks;     // as SeqTiles
  int heads, last_head;              // heads of a group, and the last one of this group: see below
  int tile0, n_seg, n_tiles;         // first tile, tiles, and those of them that hold keys of its rows (at least one)
  int keys;                          // cached tokens and rows up to its last one
  const uint8_t *k_cache, *k_rows;   // of the head
};

// This workgroup's tiles: an equal share of all, in the order sequence, group of heads, block, head, tile.  A group has as
// many heads as a share holds units: the blocks of a head, which read the same keys, then run beside each other on one XCD
// (consecutive shares do) and not one after the other in one workgroup.  Batch of 32, 8 key/value heads of 128, 360 query rows
// a head in three blocks: 298 us with all tiles of a block before the next one's (940 MB from beyond the L2 for 385 MB of keys
// and values) and no unit cost, 244 us so.
template <int BM, int COST>
struct Schedule {
  const AttentionJob& p;
  const int G;
  uint64_t all, groups, at, end, start;   // cost of all; workgroups that share it; this one's places; where sequence q starts
  uint64_t unit_end;                      // of the segment that is worked on
  int me, share, q;

  // false: this workgroup has no share
  __device__ __forceinline__ bool live(const AttentionSpace& ws) {
    const int lane = threadIdx.x & 63;
    // costs of 64 sequences, and of each with those before it
    auto costs = [&](int q0, uint64_t& t, uint64_t& sum) {
      t = sum = q0 + lane < p.batch ? seq_tiles(p, q0 + lane, BM, COST).total : 0;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const uint64_t y = __shfl_up((unsigned long long)sum, d);
        if (lane >= d) sum += y;
      }
    };
    uint64_t t0, sum0;
    costs(0, t0, sum0);
    all = __shfl((unsigned long long)sum0, 63);
    for (int q0 = 64; q0 < p.batch; q0 += 64) {
      uint64_t t, sum;
      costs(q0, t, sum);
      all += __shfl((unsigned long long)sum, 63);
    }
    all = uniform(all);
    groups = min((uint64_t)(all <= kFewCost * 256 ? 256 : ws.groups), (all + ws.least - 1) / ws.least);
    // (workgroups go round the XCDs: these are as many on each, whatever their number)
    const int per_xcd = ((int)groups + 7) / 8;
    me = (int)(blockIdx.x % 8) * per_xcd + (int)(blockIdx.x / 8);
    if (blockIdx.x == 0 && threadIdx.x == 0) *ws.live = (int)groups;
    if ((int)(blockIdx.x / 8) >= per_xcd || me >= (int)groups) return false;
    at = uniform(all * me / groups);
    end = uniform(all * (me + 1) / groups);
    share = uniform((int)min(all / groups, (uint64_t)(1 << 30)));
    q = 0;
    start = 0;
    for (int q0 = 0; q0 < p.batch; q0 += 64) {   // (lengths that change under way end the search, and the work, early)
      uint64_t t = t0, sum = sum0;
      if (q0 > 0) costs(q0, t, sum);
      const uint64_t over = __ballot(start + sum > at);
      if (over) {
        const int l = __ffsll((unsigned long long)over) - 1;
        q = uniform(q0 + l);
        start = uniform(start + (uint64_t)__shfl((unsigned long long)(sum - t), l));
        return true;
      }
      start = uniform(start + (uint64_t)__shfl((unsigned long long)sum, 63));
    }
    q = p.batch;
    return true;
  }

  __device__ __forceinline__ uint64_t of_sequence(Segment& s, int seq) const {
    const SeqTiles t = seq_tiles<true>(p, seq, BM, COST);
    s.q = seq, s.ctx = t.ctx, s.nodes = t.nodes, s.tiles = t.tiles, s.blocks = t.blocks;
    s.heads = uniform(min(max(share / (t.tiles + COST), 1), p.kv_heads));
    return t.total;
  }
  // the rest of a segment, `cost` of whose unit other workgroups bear, from place `from` on; false: there is no tile in it
  __device__ __forceinline__ bool finish(Segment& s, uint64_t from, int cost) const {
    const int upto = cost + (int)min(end - from, (uint64_t)(s.tiles + COST - cost));
    s.tile0 = max(cost - COST, 0);
    s.n_seg = max(upto - COST, 0) - s.tile0;
    s.keys = s.ctx + min(s.nodes, (s.block * BM + BM - 1) / G) + 1;
    s.n_tiles = max(min(s.n_seg, (s.keys + KT - 1) / KT - s.tile0), 1);   // (tiles behind that hold rows that are nobody's ancestor)
    s.k_cache = static_cast<const uint8_t*>(p.k) + (int64_t)s.g * p.cache_head;
    s.k_rows = static_cast<const uint8_t*>(p.k_new) + s.q * p.new_seq + (int64_t)s.g * p.new_head;
    return s.n_seg > 0;
  }
  // the segment behind s, the one that is worked on; false: there is none
  __device__ __forceinline__ bool following(Segment& s) const {
    if (unit_end >= end) return false;
    if (s.g < s.last_head) {
      ++s.g;
    } else if (++s.block < s.blocks) {
      s.g -= (s.g % s.heads);   // (groups start at multiples of their size)
    } else {
      s.block = 0;
      if (++s.g == p.kv_heads) {
        s.g = 0;
        do {
          if (++s.q >= p.batch) return false;
        } while (of_sequence(s, s.q) == 0);
      }
      s.last_head = min(s.g + s.heads, p.kv_heads) - 1;
    }
    return finish(s, unit_end, 0);
  }
  __device__ __forceinline__ void advance(const Segment& s) { unit_end += (uint64_t)(s.tiles + COST); }
  __device__ __forceinline__ bool first(Segment& s) {
    if (q >= p.batch || of_sequence(s, q) == 0) return false;
    const int span = s.tiles + COST;
    const uint64_t unit = uniform((at - start) / (uint64_t)span);
    const int cost = uniform((int)(at - start - unit * (uint64_t)span));
    const int per = s.heads * s.blocks, group = uniform((int)(unit / (uint64_t)per)), in = uniform((int)(unit - (uint64_t)group * (uint64_t)per));
    s.last_head = min((group + 1) * s.heads, p.kv_heads) - 1;
    const int size = s.last_head + 1 - group * s.heads;
    s.block = uniform(in / size);
    s.g = uniform(group * s.heads + in - s.block * size);
    unit_end = at + (uint64_t)(span - cost);
    if (finish(s, at, cost)) return true;
    if (!following(s)) return false;   // (nothing but the cost of its queries)
    advance(s);
    return true;
  }
  // the workgroup that takes the last tile of the segment's unit
  __device__ __forceinline__ int last() const { return (int)((unit_end * groups - 1) / all); }
};

// A workgroup's share, by Copy's way of bringing tiles into LDS.
template <bool BF16, int DP, int MQ, int WK, typename Copy>
__device__ __forceinline__ void attention_body(const AttentionJob& p, const AttentionSpace& ws, uint8_t* smem, uint32_t (*s_valid)[4], uint32_t& s_again) {
  typedef AttentionShape<BF16, DP, MQ, WK> S;
  typedef AttentionTile<BF16, DP, MQ, WK> Tile;
  constexpr int ESZ = S::ESZ, BM = S::BM;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, grp = lane >> 4;
  const int wq = wave / WK, wk = wave % WK;
  const int G = p.q_heads / p.kv_heads;

  Schedule<BM, unit_cost(BF16)> plan = {p, G};
  if (!plan.live(ws)) return;
  Segment now;
  Owner mine = {-1, 0, 0, 0, 0};
  bool more = plan.first(now);
  if (!more) {
    if (tid == 0) ws.owner[plan.me] = mine;
    return;
  }
  const int me = plan.me;

  // a negative scale goes into the queries' sign, a scale of zero makes them zero: the largest product has the largest weight
  const float q_sign = p.scale < 0 ? -1.0f : p.scale == 0 ? 0.0f : 1.0f;
  const float sc = (p.scale == 0 ? 1.0f : fabsf(p.scale)) * kLog2e;
  const int last_word = p.head_dim * ESZ / 16 - 1;

  Copy copy = {p, s_valid, last_word, static_cast<const uint8_t*>(p.v) - static_cast<const uint8_t*>(p.k),
               static_cast<const uint8_t*>(p.v_new) - static_cast<const uint8_t*>(p.k_new)};
  copy.init();
  bool fresh = true;   // (kEarly) nothing has been requested beyond tile 0
  typename Copy::Places f = copy.places(now, 0), f_next = {-1, 0};
  copy.copy(copy.source(now, 0, f), (lds_u8*)smem, s_valid[0]);
  typename Copy::Source up = Copy::nothing();   // what is copied next
  int turn = 0, n_units = 0;   // tiles and segments so far: which buffers are in use
  bool careful = false;        // the second pass over this share
  // The first segment whose sums in this wave are not finite, and the first of this pass: the wave has written its outputs before that
  // one in the first pass, and writes the others in the second (out may be q: what is read again has not been written).
  int first_odd = 1 << 30, unit0 = 0;
  if (tid == 0) s_again = 0;
  while (more) {
    Segment next = now;
    more = plan.following(next);
    const int rows = (now.nodes + 1) * G - now.block * BM;                     // query rows from this unit's first on
    // ---- parents' rows, where tiles hold rows (two sets: others may still be at the last segment) ----
    uint16_t* s_up = reinterpret_cast<uint16_t*>(smem + S::LDS) + (n_units & 1) * ((p.M + 8) & ~7);
    if ((now.tile0 + now.n_tiles) * KT > now.ctx)
      for (int i = tid; i < now.keys - now.ctx - 1; i += 256) {
        const int up = p.node_parent[(int64_t)now.q * p.M + i];
        s_up[i + 1] = (uint16_t)(up >= 0 && up < i ? up + 1 : 0);
      }
    // ---- queries ----
    Tile x;
#pragma unroll
    for (int mq = 0; mq < MQ; ++mq) {
      const int m = (wq * MQ + mq) * 16 + l16, mm = m < rows ? now.block * BM + m : 0;
      x.row_of[mq] = mm / G;
      const uint8_t* from = static_cast<const uint8_t*>(p.q) + now.q * p.q_seq + (int64_t)x.row_of[mq] * p.q_row + (int64_t)(now.g * G + mm % G) * p.q_head;
#pragma unroll
      for (int s = 0; s < Tile::QS; ++s) {
        const int word = s * 4 + grp;
        u32x4 raw = {0, 0, 0, 0};
        if (word <= last_word) raw = *reinterpret_cast<const u32x4*>(from + word * 16);
        if (q_sign != 1.0f) {
#pragma unroll
          for (int i = 0; i < 4; ++i) raw[i] = q_sign == 0.0f ? 0u : raw[i] ^ (BF16 ? 0x80008000u : 0x80000000u);
        }
        x.qf[mq][s] = __builtin_bit_cast(typename Tile::qword, raw);
      }
      x.m_run[mq] = kLowest;
      x.l_run[mq] = 0;
#pragma unroll
      for (int d = 0; d < DP / 16; ++d) x.o[mq][d] = (f32x4){0, 0, 0, 0};
    }
    typename Copy::Source first = Copy::nothing();   // of the next segment
    if (more) f_next = copy.places(next, 0);
    if constexpr (Copy::kEarly) {
      if (now.n_tiles == 1) up = more ? copy.source(next, 0, f_next) : first;
      else if (fresh) up = copy.source(now, 1, f);
      fresh = false;
    } else {
      if (more) first = copy.source(next, 0, f_next);
      if (now.n_tiles > 1) up = copy.source(now, 1, f);
      else up = first;
    }

    bool odd = last_word < S::CH - 1;
    const bool active = uniform(wq) * MQ * 16 < rows;   // (of a unit with few rows only the first waves have any: the others just copy)
    // ---- tiles.  The next one is copied into the other buffer while one is worked on; the two buffers are distinct objects to
    // the compiler (restrict), so that a read of one does not wait for the copies into the other ----
    auto tile = [&](lds_u8* cur, lds_u8* other, int t) {
      attention_turn<BF16, DP, MQ, WK>(
          x, cur, other, s_valid[turn & 1], (now.tile0 + t) * KT, now.ctx, s_up, sc, active, careful, last_word, odd, [&] { copy.landed(); },
          [&](lds_u8* to) {
            if (up.k_cache) copy.copy(up, to, s_valid[(turn + 1) & 1]);
          },
          [&] {
            if constexpr (Copy::kEarly) {
              if (t + 2 < now.n_tiles) up = copy.source(now, t + 2, f);
              else if (!more || (t + 1 == now.n_tiles && next.n_tiles == 1)) up = Copy::nothing();
              else up = copy.source(next, t + 2 - now.n_tiles, f_next);
            }
          });
      if constexpr (!Copy::kEarly) {
        if (t + 2 < now.n_tiles) up = copy.source(now, t + 2, f);
        else up = first;
      }
      ++turn;
    };
    for (int t = 0; t < now.n_tiles;) {
      if (turn & 1) tile((lds_u8*)(smem + S::LDS / 2), (lds_u8*)smem, t++);
      if (t < now.n_tiles && !(turn & 1)) tile((lds_u8*)smem, (lds_u8*)(smem + S::LDS / 2), t++);
    }
#pragma unroll
    for (int mq = 0; mq < MQ; ++mq) x.l_run[mq] = groups_sum(x.l_run[mq]);

    // ---- join of the waves that took other keys of the same rows, through the buffer of the last tile ----
    if constexpr (WK > 1) {
      float* box = reinterpret_cast<float*>(smem + ((turn - 1) & 1) * (S::LDS / 2));
      constexpr int PER = MQ * (DP / 4 + 2);   // values per lane
      __syncthreads();
      if (wk > 0) {
        float* to = box + ((wk - 1) * S::WQ + wq) * PER * 64 + lane;
#pragma unroll
        for (int mq = 0; mq < MQ; ++mq) {
          to[(mq * (DP / 4 + 2)) * 64] = x.m_run[mq];
          to[(mq * (DP / 4 + 2) + 1) * 64] = x.l_run[mq];
#pragma unroll
          for (int d = 0; d < DP / 16; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) to[(mq * (DP / 4 + 2) + 2 + d * 4 + i) * 64] = x.o[mq][d][i];
        }
      }
      __syncthreads();
      if (wk == 0) {
        for (int w = 0; w < WK - 1; ++w) {
          const float* from = box + (w * S::WQ + wq) * PER * 64 + lane;
#pragma unroll
          for (int mq = 0; mq < MQ; ++mq) {
            const float m = from[(mq * (DP / 4 + 2)) * 64], m_new = fmaxf(m, x.m_run[mq]);
            const float mine_ = __builtin_amdgcn_exp2f(x.m_run[mq] - m_new), its = __builtin_amdgcn_exp2f(m - m_new);
            x.m_run[mq] = m_new;
            x.l_run[mq] = x.l_run[mq] * mine_ + from[(mq * (DP / 4 + 2) + 1) * 64] * its;
#pragma unroll
            for (int d = 0; d < DP / 16; ++d)
#pragma unroll
              for (int i = 0; i < 4; ++i) x.o[mq][d][i] = x.o[mq][d][i] * mine_ + from[(mq * (DP / 4 + 2) + 2 + d * 4 + i) * 64] * its;
          }
        }
      }
    }

    // ---- out, or what has been summed so far ----
    const bool whole = now.n_seg == now.tiles;
    if (!whole && now.tile0 == 0)   // (the unit ends in the workgroup that takes its last tile)
      mine = {now.q, now.g, now.block, plan.last(), min(rows, BM)};
    if (odd && !careful) {
      float zero = 0;
#pragma unroll
      for (int mq = 0; mq < MQ; ++mq)
#pragma unroll
        for (int d = 0; d < DP / 16; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) zero = __builtin_fmaf(x.o[mq][d][i], 0.0f, zero);
      if (wk == 0 && __any(!(zero == 0.0f))) {
        if (lane == 0) s_again = 1;
        first_odd = min(first_odd, n_units);
      }
    }
    if (careful && wk == 0 && (now.tile0 + now.n_tiles) * KT > now.ctx)
      add_left_out(x, now.k_rows, copy.to_v_rows, p.new_row, now.ctx, now.tile0 * KT, (now.tile0 + now.n_tiles) * KT, s_up, last_word);
    if (wk == 0 && (careful ? n_units - unit0 >= first_odd : n_units < first_odd)) {
#pragma unroll
      for (int mq = 0; mq < MQ; ++mq) {
        const int m = (wq * MQ + mq) * 16 + l16;
        if (m < rows) {
          if (whole) {
            const float inv = 1.0f / x.l_run[mq];
            uint8_t* to = static_cast<uint8_t*>(p.out) + now.q * p.out_seq + (int64_t)x.row_of[mq] * p.out_row + (int64_t)(now.g * G + (now.block * BM + m) % G) * p.out_head;
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) {
              const int e = d * 16 + grp * 4;
              if (e < p.head_dim) {
                const f32x4 v = x.o[mq][d] * inv;
                if constexpr (BF16) *reinterpret_cast<uint64_t*>(to + e * 2) = (uint64_t)f32_to_bf16_pair(v[2], v[3]) << 32 | f32_to_bf16_pair(v[0], v[1]);
                else *reinterpret_cast<f32x4*>(to + e * 4) = v;
              }
            }
          } else {
            float* to = ws.part + ((int64_t)(me * 2 + (now.tile0 == 0 ? 1 : 0)) * BM + m) * (DP + 4);
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) *reinterpret_cast<f32x4*>(to + d * 16 + grp * 4) = x.o[mq][d];
            if (grp == 0) to[DP] = x.m_run[mq], to[DP + 1] = x.l_run[mq];
          }
        }
      }
    }
    plan.advance(next);
    now = next;
    f = f_next;
    ++n_units;
    if (!more && !careful) {
      __syncthreads();
      if (s_again) {
        careful = true;
        unit0 = n_units;
        more = plan.first(now);
        f = copy.places(now, 0);
        fresh = true;
        copy.copy(copy.source(now, 0, f), (lds_u8*)(smem + (turn & 1) * (S::LDS / 2)), s_valid[turn & 1]);
      }
    }
  }
  if (tid == 0) ws.owner[me] = mine;
}

// Units that several workgroups took part in: workgroup (w, y) joins some query rows of the one that started in workgroup w of
// the launch above, in the order of the keys.  One small call (32 heads of 34 query rows, 6 parts each) reads and writes as
// much for its parts as for its keys and values: the rows are spread over as many workgroups as there are.
constexpr int join_rows(int DP) { return 256 / (DP / 4); }
template <bool BF16, int DP, int BM>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionJob p, AttentionSpace ws) {
  const int w = blockIdx.x, tid = threadIdx.x, G = p.q_heads / p.kv_heads;
  const Owner u = ws.owner[w];
  const int live = *ws.live;
  constexpr int PER = DP / 4;   // threads of a row
  const int m = blockIdx.y * join_rows(DP) + tid / PER, e = tid % PER * 4, mm = u.block * BM + m;
  if (w >= live || u.q < 0 || m >= u.rows || e >= p.head_dim) return;
  f32x4 o = {0, 0, 0, 0};
  float top = kLowest, l = 0;
  // eight parts' loads at a time: one after the other they wait for each other's latency
  for (int x0 = w; x0 <= u.last; x0 += 8) {
    f32x4 po[8];
    f32x2 pm[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int x = min(x0 + j, u.last);
      const float* from = ws.part + ((int64_t)(x * 2 + (x == w ? 1 : 0)) * BM + m) * (DP + 4);
      po[j] = *reinterpret_cast<const f32x4*>(from + e);
      pm[j] = *reinterpret_cast<const f32x2*>(from + DP);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (x0 + j > u.last) break;
      const float m_new = fmaxf(top, pm[j][0]), keep = __builtin_amdgcn_exp2f(top - m_new), add = __builtin_amdgcn_exp2f(pm[j][0] - m_new);
      o = o * keep + po[j] * add;
      l = l * keep + pm[j][1] * add;
      top = m_new;
    }
  }
  const float inv = 1.0f / l;
  o = o * inv;
  uint8_t* to = static_cast<uint8_t*>(p.out) + u.q * p.out_seq + (int64_t)(mm / G) * p.out_row + (int64_t)(u.g * G + mm % G) * p.out_head;
  if constexpr (BF16) *reinterpret_cast<uint64_t*>(to + e * 2) = (uint64_t)f32_to_bf16_pair(o[2], o[3]) << 32 | f32_to_bf16_pair(o[0], o[1]);
  else *reinterpret_cast<f32x4*>(to + e * 4) = o;
}

constexpr int kWideRows = 16;   // query rows of a unit of float32 heads of more than 128 elements

// Query rows of a key/value head: at most 16, the waves share the keys; at most 32, by twos; more, each has rows of its own.
struct AttentionPlan {
  int dp, bm, groups, least;
};
inline AttentionPlan plan_attention(int M, int q_heads, int kv_heads, int head_dim, bool bf16) {
  AttentionPlan a;
  a.dp = head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256;
  const int64_t rows = (int64_t)(M + 1) * (q_heads / kv_heads);
  a.bm = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 || a.dp == 256 || !bf16 ? 64 : 128;
  a.groups = a.dp * (bf16 ? 1 : 2) <= 128 ? 512 : 256;   // two workgroups of 64 KiB fit a CU
  if (!bf16 && a.dp == 256) a.bm = kWideRows, a.groups = 512;
  a.least = 2;
  return a;
}

inline int64_t owner_bytes(int groups) { return ((int64_t)groups * sizeof(Owner) + 16 + 255) & ~(int64_t)255; }

inline AttentionSpace space_of(const AttentionJob& job, const AttentionPlan& plan) {
  AttentionSpace ws;
  ws.live = static_cast<int*>(job.workspace);
  ws.owner = reinterpret_cast<Owner*>(ws.live + 4);
  ws.part = reinterpret_cast<float*>(static_cast<uint8_t*>(job.workspace) + owner_bytes(plan.groups));
  ws.groups = plan.groups;
  ws.least = plan.least;
  return ws;
}

}  // namespace specdraft
