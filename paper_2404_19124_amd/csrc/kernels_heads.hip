// Rows of heads on their way: norms of queries and keys for each head, the position rotation, and keys and values into a cache of the
// same type or of four bits.
//   n = x * (1 / sqrt(mean(x^2) + eps)) * weight;  of a pair (a, b) of elements with the angle of its position: (a cos - b sin, b cos + a sin)
// The mean and its root are 64-bit numbers, rounded to float32 as a factor; every other operation is float32 and rounded by itself, so that
// what is stored does not hang on the compiler's choice of fused operations (in a cache of four bits one rounding more or less is a
// third of a value); one rounding to the rows' type follows.
#include <type_traits>

#include "device_utils.h"
#include "packed.h"
#include "rows_internal.h"
#include "spec_internal.h"

namespace specdraft {

// One 16-byte word of a row: E elements in float32.
template <bool BF16>
struct HeadWord {
  static constexpr int E = BF16 ? 8 : 4;
  float x[E];
  __device__ __forceinline__ void from(u32x4 raw) {
#pragma unroll
    for (int i = 0; i < E; ++i) {
      if constexpr (BF16) x[i] = bf16_bits_to_f32(raw[i / 2] >> (i & 1) * 16 & 0xffffu);
      else x[i] = __uint_as_float(raw[i]);
    }
  }
  __device__ __forceinline__ u32x4 raw() const {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) r[i] = f32_to_bf16_pair(x[2 * i], x[2 * i + 1]);
      else r[i] = __float_as_uint(x[i]);
    }
    return r;
  }
  __device__ __forceinline__ double squares() const {
    double s = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) s += (double)x[i] * (double)x[i];
    return s;
  }
  __device__ __forceinline__ void load(const float* at) {
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(at + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[i + j] = v[j];
    }
  }
  __device__ __forceinline__ void scale(float inv, const HeadWord& weight) {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = x[i] * inv * weight.x[i];
  }
};

__device__ __forceinline__ float head_factor(double squares, int head_dim, double eps) { return (float)(1.0 / sqrt(squares / head_dim + eps)); }

// words whose elements are the first and the second ones of pairs
template <bool BF16>
__device__ __forceinline__ void turn(HeadWord<BF16>& a, HeadWord<BF16>& b, const HeadWord<BF16>& c, const HeadWord<BF16>& s) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < HeadWord<BF16>::E; ++i) {
    const float x = a.x[i] * c.x[i] - b.x[i] * s.x[i], y = b.x[i] * c.x[i] + a.x[i] * s.x[i];
    a.x[i] = x, b.x[i] = y;
  }
}
// a word of neighbours that are pairs, with the first E / 2 angles of c and s
template <bool BF16>
__device__ __forceinline__ void turn_pairs(HeadWord<BF16>& a, const HeadWord<BF16>& c, const HeadWord<BF16>& s) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < HeadWord<BF16>::E; i += 2) {
    const float x = a.x[i] * c.x[i / 2] - a.x[i + 1] * s.x[i / 2], y = a.x[i + 1] * c.x[i / 2] + a.x[i] * s.x[i / 2];
    a.x[i] = x, a.x[i + 1] = y;
  }
}
template <bool BF16>
__device__ __forceinline__ void load_half(HeadWord<BF16>& w, const float* at) {   // E / 2 of them
  constexpr int H = HeadWord<BF16>::E / 2;
#pragma unroll
  for (int i = 0; i < H; ++i) w.x[i] = at[i];
}

// sum over `width` neighbouring lanes, a power of two
__device__ __forceinline__ double lanes_sum(double x, int width) {
  for (int d = 1; d < width; d *= 2) x += __shfl_xor(x, d);
  return x;
}

// Where an entry's rows come from and go to, and its position; false: nothing is done for it.
template <bool APPEND>
__device__ __forceinline__ bool entry_of(const HeadsJob& p, int t, int64_t (&from)[2], int64_t (&to)[2], int& pos) {
  if constexpr (APPEND) {
    const int layer = blockIdx.z, slot = p.slot[t], src = p.src_row ? p.src_row[t] : t;
    pos = p.cos ? p.pos[t] : 0;
    if (slot < 0 || slot >= p.n_slots || src < 0 || src >= p.rows) return false;
    const int b = slot / p.block_size;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      from[i] = layer * p.side[i].from_far + src * p.side[i].from_row;
      to[i] = layer * p.side[i].to_far + b * p.side[i].to_block + (slot - b * p.block_size) * p.side[i].to_row;
    }
  } else {
    const int R = p.M + 1, q = t / R, r = t - q * R;
    if (p.pos) {
      pos = p.pos[t];
      if (pos < 0) return false;
    } else {
      const int nodes = p.n_nodes ? min(max(p.n_nodes[q], -1), p.M) : p.M;
      if (r > nodes) return false;
      pos = p.cos ? p.ctx_len[q] + (r ? p.node_depth[(int64_t)q * p.M + r - 1] : 0) : 0;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      from[i] = q * p.side[i].from_far + r * p.side[i].from_row;
      to[i] = q * p.side[i].to_far + r * p.side[i].to_row;
    }
  }
  return !p.cos || (pos >= 0 && pos < p.n_pos);
}

// A wave takes heads of one entry, `lanes` lanes to a head.  A lane holds the words of the first and of the second elements of its pairs
// (so a head's row is read once, and may be written where it was read), or one word.
template <bool BF16, bool PAIRS, bool APPEND>
__global__ __launch_bounds__(256) void heads_kernel(HeadsJob p) {
  typedef HeadWord<BF16> Word;
  const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= p.entries) return;
  int64_t from[2], to[2];
  int pos;
  if (!entry_of<APPEND>(p, t, from, to, pos)) return;
  const int slot = lane & (p.lanes - 1), per = 64 / p.lanes, words = p.row_words, half = PAIRS ? 0 : p.half_words;
  const bool active = slot < words - half, two = !PAIRS && slot < half, turned = PAIRS ? slot < p.half_words * 2 : two;
  const int a_at = two || PAIRS ? slot : slot + half, b_at = slot + half;
  Word c, s;
  if (turned) {
    const int64_t at = (int64_t)pos * p.half_words * Word::E + (PAIRS ? slot * (Word::E / 2) : slot * Word::E);
    if constexpr (PAIRS) load_half<BF16>(c, p.cos + at), load_half<BF16>(s, p.sin + at);
    else c.load(p.cos + at), s.load(p.sin + at);
  }
  const int first_trips = (p.side[0].heads + per - 1) / per, trips = first_trips + (p.side[1].heads + per - 1) / per;
  for (int trip = blockIdx.y * p.trips; trip < min(trips, (int)(blockIdx.y + 1) * p.trips); ++trip) {
    const bool second = trip >= first_trips;   // (a trip's heads are all of one side: its fields are scalars)
    const HeadSide& side = second ? p.side[1] : p.side[0];
    const int head = (second ? trip - first_trips : trip) * per + lane / p.lanes;
    const bool mine = active && head < side.heads;
    u32x4 ra = {0, 0, 0, 0}, rb = {0, 0, 0, 0};
    const uint8_t* src = side.from + (second ? from[1] : from[0]) + head * side.from_head;
    if (mine) ra = *reinterpret_cast<const u32x4*>(src + a_at * 16);
    if (mine && two) rb = *reinterpret_cast<const u32x4*>(src + b_at * 16);
    Word a, b;
    a.from(ra), b.from(rb);
    if (side.weight) {
      const float inv = head_factor(lanes_sum(a.squares() + b.squares(), p.lanes), p.head_dim, p.eps);
      const float* w = side.weight + (APPEND ? (int64_t)blockIdx.z * p.head_dim : 0);
      Word x;
      if (active) x.load(w + a_at * Word::E), a.scale(inv, x);
      if (two) x.load(w + b_at * Word::E), b.scale(inv, x);
    }
    if (turned && side.turned) {
      if constexpr (PAIRS) turn_pairs<BF16>(a, c, s);
      else turn<BF16>(a, b, c, s);
    }
    uint8_t* dst = side.to + (second ? to[1] : to[0]) + head * side.to_head;
    if (mine) *reinterpret_cast<u32x4*>(dst + a_at * 16) = a.raw();
    if (mine && two) *reinterpret_cast<u32x4*>(dst + b_at * 16) = b.raw();
  }
}

static int power_of_two(int n) {
  int p = 1;
  while (p < n) p *= 2;
  return p;
}

// of `trips` for each of so many entries: few entries have theirs spread over several waves
static int trips_of_a_wave(int trips, int64_t entries) {
  const int parts = (int)min((int64_t)trips, max((int64_t)1, 4096 / entries));
  return (trips + parts - 1) / parts;
}

hipError_t launch_heads(HeadsJob job, bool bf16, bool append, hipStream_t st) {
  job.lanes = power_of_two(job.row_words - (job.pairs ? 0 : job.half_words));
  const int per = 64 / job.lanes, trips = (job.side[0].heads + per - 1) / per + (job.side[1].heads + per - 1) / per;
  job.trips = trips_of_a_wave(trips, (int64_t)job.entries * job.layers);
  const dim3 grid((unsigned)((job.entries + 3) / 4), (unsigned)((trips + job.trips - 1) / job.trips), (unsigned)job.layers);
#define LAUNCH(BF16, PAIRS, APPEND) \
  if (bf16 == BF16 && (job.pairs != 0) == PAIRS && append == APPEND) hipLaunchKernelGGL((heads_kernel<BF16, PAIRS, APPEND>), grid, dim3(256), 0, st, job)
  LAUNCH(true, false, false);
  LAUNCH(true, true, false);
  LAUNCH(false, false, false);
  LAUNCH(false, true, false);
  LAUNCH(true, false, true);
  LAUNCH(true, true, true);
  LAUNCH(false, false, true);
  LAUNCH(false, true, true);
#undef LAUNCH
  return hipGetLastError();
}

// ---- a cache of four bits --------------------------------------------------------------------------------------
// A group of 32 elements has a scale 2^e, e the smallest with (largest amount) <= 7 * 2^e, within [-125, 125]: what is above 6 * 2^e is
// then off by half a step at most, as if the amounts went on.  Codes are rounded to the nearest amount, of two as near to the even code.

// Scale byte of a group, four lanes with eight elements each, and the codes of this lane's.
__device__ __forceinline__ uint32_t pack_group(const float (&x)[8], uint32_t& codes) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xb1, 0xf, 0xf, true));   // lanes 1 0 3 2 of the four
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4e, 0xf, 0xf, true));   // lanes 2 3 0 1
  codes = 0;
  if (top >= 0x7f800000u) return 255;   // an infinity or NaN: no element of the group is a number
  const int e = min(max((int)(top >> 23) - 129 + ((top & 0x7fffffu) > 0x600000u), -125), 125);
  const float scale = __uint_as_float((uint32_t)(e + 127) << 23);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
  return (uint32_t)(e + 127);
}

// A lane takes a word of a head, eight elements, four lanes a group of 32: a wave reads 1 KiB and writes 256 bytes in a row.  The other
// elements of its pairs it reads again, from the cache where its neighbours' reads have brought them, and norms and turns them too: 16,000
// tokens of 8 heads of 128 with their norms, rotation and tables, 91 MB, 26 us, 3.5 TB/s (a whole group to a lane, 64 bytes apart: 53 us).  Vector
// instructions take 63 % of the SIMDs' time and 48 % of the waves' is waiting: both bound it (rows into a cache of 16 bits: 28 and 71 %, 5.0 TB/s).
template <bool PAIRS>
__global__ __launch_bounds__(256) void pack_kernel(PackJob p) {
  typedef HeadWord<true> Word;
  const int lane = threadIdx.x & 63, t = blockIdx.x * 4 + (threadIdx.x >> 6), layer = blockIdx.z;
  if (t >= p.entries) return;
  const int slot = p.slot[t], src = p.src_row ? p.src_row[t] : t, pos = p.cos ? p.pos[t] : 0;
  if (slot < 0 || slot >= p.n_slots || src < 0 || src >= p.rows || (p.cos && (pos < 0 || pos >= p.n_pos))) return;
  const int block = slot / p.block_size, in = slot - block * p.block_size;
  const int word = lane & (p.lanes - 1), per = 64 / p.lanes;
  const bool active = word < p.groups * 4, turned = word < 2 * p.half_words, first = word < p.half_words;
  const int other = !turned || PAIRS ? word : first ? word + p.half_words : word - p.half_words;
  Word c, s;
  if (turned) {
    const int64_t at = (int64_t)pos * p.half_words * 8;
    if constexpr (PAIRS) load_half<true>(c, p.cos + at + word * 4), load_half<true>(s, p.sin + at + word * 4);
    else c.load(p.cos + at + min(word, other) * 8), s.load(p.sin + at + min(word, other) * 8);
  }
  const int side_trips = (p.heads + per - 1) / per;
  for (int trip = blockIdx.y * p.trips; trip < min(2 * side_trips, (int)(blockIdx.y + 1) * p.trips); ++trip) {
    const bool key = trip < side_trips;
    const int head = (key ? trip : trip - side_trips) * per + lane / p.lanes;
    const bool mine = active && head < p.heads;
    const uint8_t* from = (key ? p.k_new : p.v_new) + layer * p.new_layer + src * p.new_row + head * p.new_head;
    u32x4 rx = {0, 0, 0, 0}, ry = {0, 0, 0, 0};
    if (mine) rx = *reinterpret_cast<const u32x4*>(from + word * 16);
    if (!PAIRS && mine && key && turned) ry = *reinterpret_cast<const u32x4*>(from + other * 16);
    Word x, y;
    x.from(rx), y.from(ry);
    if (p.weight && key) {
      const float inv = head_factor(lanes_sum(x.squares(), p.lanes), p.groups * 32, p.eps);
      const float* weight = p.weight + (int64_t)layer * p.groups * 32;
      Word w;
      if (active) w.load(weight + word * 8), x.scale(inv, w);
      if (!PAIRS && active && turned) w.load(weight + other * 8), y.scale(inv, w);
    }
    if (turned && key) {
      if constexpr (PAIRS) turn_pairs<true>(x, c, s);
      else if (first) turn<true>(x, y, c, s);
      else turn<true>(y, x, c, s);
    }
    uint32_t codes;
    const uint32_t scale = pack_group(x.x, codes);
    const int64_t to = layer * p.layer + block * p.block + in * p.slot_stride + head * p.head + word * 4;
    const int64_t at = layer * p.scale_layer + block * p.scale_block + in * p.scale_slot + head * p.scale_head + word / 4;
    if (mine) *reinterpret_cast<uint32_t*>((key ? p.k : p.v) + to) = codes;
    if (mine && word % 4 == 0) (key ? p.k_scale : p.v_scale)[at] = (uint8_t)scale;
  }
}

hipError_t launch_pack(PackJob job, hipStream_t st) {
  job.lanes = power_of_two(job.groups * 4);
  const int per = 64 / job.lanes, trips = 2 * ((job.heads + per - 1) / per);
  job.trips = trips_of_a_wave(trips, (int64_t)job.entries * job.layers);
  const dim3 grid((unsigned)((job.entries + 3) / 4), (unsigned)((trips + job.trips - 1) / job.trips), (unsigned)job.layers);
  if (job.pairs) hipLaunchKernelGGL((pack_kernel<true>), grid, dim3(256), 0, st, job);
  else hipLaunchKernelGGL((pack_kernel<false>), grid, dim3(256), 0, st, job);
  return hipGetLastError();
}

// Eight elements of a key and of a value per thread and turn.  What bounds it is memory, 3.8 bytes written for each one read: stores that the
// caches do not keep take 60,000 tokens of 8 heads of 128 from 76 to 52 us (4.1 -> 6.0 TB/s), with a reader of the rows behind it from 76 to
// 66 us at 125 MiB and from 163 to 160 at 250; below 32 MiB the two are the same.  (Rows rotated so are faster by themselves, 42 -> 41 us at
// 125 MiB, but with their reader slower, 81 -> 92.)
__global__ __launch_bounds__(256) void unpack_kernel(UnpackJob p) {
  const int per = p.heads * p.groups * 4, layer = blockIdx.y;
  const int64_t total = (int64_t)p.count * per;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int t = (int)(i / per), w = (int)(i - (int64_t)t * per), h = w / (p.groups * 4), c = w - h * (p.groups * 4);
    const int slot = p.slot[t];
    if (slot < 0 || slot >= p.n_slots) continue;
    const int block = slot / p.block_size, in = slot - block * p.block_size;
    const int64_t from = layer * p.layer + block * p.block + in * p.slot_stride + h * p.head + c * 4;
    const int64_t at = layer * p.scale_layer + block * p.scale_block + in * p.scale_slot + h * p.scale_head + c / 4;
    const int64_t to = layer * p.out_layer + t * p.out_row + h * p.out_head + c * 16;
    __builtin_nontemporal_store(unpack_word(*reinterpret_cast<const uint32_t*>(p.k + from), p.k_scale[at]), reinterpret_cast<u32x4*>(p.k_out + to));
    __builtin_nontemporal_store(unpack_word(*reinterpret_cast<const uint32_t*>(p.v + from), p.v_scale[at]), reinterpret_cast<u32x4*>(p.v_out + to));
  }
}

hipError_t launch_unpack(const UnpackJob& job, hipStream_t st) {
  const int64_t words = (int64_t)job.count * job.heads * job.groups * 4, groups = (words + 255) / 256;
  hipLaunchKernelGGL(unpack_kernel, dim3((unsigned)(groups < 8192 ? groups : 8192), job.layers), dim3(256), 0, st, job);
  return hipGetLastError();
}

}  // namespace specdraft
