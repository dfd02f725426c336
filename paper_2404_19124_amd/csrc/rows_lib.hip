// C ABI of the operators on the rows of a token tree (declared in include/spec.h): argument checks and launches.
#include <algorithm>
#include <initializer_list>
#include <utility>

#include "rows_internal.h"
#include "spec_internal.h"
#include "status.h"

using namespace specdraft;

static bool known_dtype(int32_t d) { return d == SPEC_F32 || d == SPEC_BF16; }
static int element_bytes(int32_t d) { return d == SPEC_BF16 ? 2 : 4; }

// every row of heads starts on a multiple of 16 bytes
static bool rows_aligned(const void* at, int64_t a, int64_t b, int64_t c, int esz) {
  return !(((uint64_t)reinterpret_cast<uintptr_t>(at) | (uint64_t)(a * esz) | (uint64_t)(b * esz) | (uint64_t)(c * esz)) & 15);
}
static bool rows_aligned(const spec_rows_t& r, int esz) { return rows_aligned(r.at, r.seq_stride, r.row_stride, r.head_stride, esz); }

// Whether no two rows of `row` elements share memory, counted along dimensions of n entries and these strides: in the order of the
// strides' sizes, each dimension's step leaves the extent of those before it behind (so do slices and permutations of a tensor)
static bool rows_apart(std::initializer_list<std::pair<int64_t, int64_t>> dims, int64_t row) {
  std::pair<__int128, int64_t> d[4];
  int n = 0;
  for (const auto& x : dims)
    if (x.first > 1) d[n++] = {x.second < 0 ? -(__int128)x.second : (__int128)x.second, x.first};
  std::sort(d, d + n);
  __int128 extent = row;
  for (int i = 0; i < n; ++i) {
    if (d[i].first < extent) return false;
    extent += d[i].first * (d[i].second - 1);
  }
  return true;
}

static spec_status_t check_heads(int32_t dtype, int32_t kv_heads, int32_t head_dim) {
  if (!known_dtype(dtype)) return fail(SPEC_EDTYPE, "dtype = %d is neither SPEC_F32 nor SPEC_BF16", dtype);
  if (kv_heads < 1 || head_dim < 1) return fail(SPEC_EINVAL, "kv_heads and head_dim must be >= 1");
  const int per = 16 / element_bytes(dtype);
  if (head_dim % per || head_dim > 256)
    return fail(SPEC_ESHAPE, "head_dim = %d must be a multiple of %d, at most 256", head_dim, per);
  return SPEC_OK;
}

static spec_status_t check_cache(const spec_cache_t& c, int esz) {
  if (!c.k || !c.v) return fail(SPEC_EINVAL, "the cache's k or v is NULL");
  if (c.n_blocks < 1 || c.block_size < 1) return fail(SPEC_EINVAL, "n_blocks and block_size must be >= 1");
  if ((int64_t)c.n_blocks * c.block_size > kMaxSlots) return fail(SPEC_ESHAPE, "n_blocks * block_size exceeds 2^30");
  if (!rows_aligned(c.k, c.block_stride, c.slot_stride, c.head_stride, esz) || (reinterpret_cast<uintptr_t>(c.v) & 15))
    return fail(SPEC_EINVAL, "rows of the cache must start on multiples of 16 bytes");
  return SPEC_OK;
}

static spec_status_t check_attention_shape(int32_t batch, int32_t M, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t dtype) {
  spec_status_t s = check_heads(dtype, kv_heads, head_dim);
  if (s != SPEC_OK) return s;
  if (batch < 1 || M < 0 || q_heads < 1) return fail(SPEC_EINVAL, "batch and q_heads must be >= 1, M >= 0");
  if (q_heads % kv_heads) return fail(SPEC_ESHAPE, "q_heads = %d is not a multiple of kv_heads = %d", q_heads, kv_heads);
  if (M > kMaxTreeItems) return fail(SPEC_ESHAPE, "M = %d exceeds %d", M, kMaxTreeItems);
  if (batch > 65535 || q_heads > 65535) return fail(SPEC_ESHAPE, "batch = %d or q_heads = %d exceeds 65535", batch, q_heads);
  return SPEC_OK;
}

extern "C" spec_status_t spec_tree_attention_workspace(int32_t batch, int32_t M, int32_t q_heads, int32_t kv_heads,
                                                       int32_t head_dim, int32_t dtype, int64_t* bytes) {
  if (!bytes) return fail(SPEC_EINVAL, "bytes is NULL");
  spec_status_t s = check_attention_shape(batch, M, q_heads, kv_heads, head_dim, dtype);
  if (s != SPEC_OK) return s;
  *bytes = attention_workspace(batch, M, q_heads, kv_heads, head_dim, dtype == SPEC_BF16);
  return SPEC_OK;
}

// What the attentions over a cache of either kind check alike, and what their jobs have in common
static spec_status_t check_attention(const spec_rows_t* q, const spec_rows_t* k_new, const spec_rows_t* v_new, const int32_t* block_table,
                                     const int32_t* ctx_len, const int32_t* node_parent, const spec_rows_t* out, int32_t batch, int32_t M,
                                     int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t dtype, int32_t block_size, int32_t max_blocks,
                                     void* workspace, int64_t workspace_bytes) {
  if (!q || !k_new || !v_new || !out || !q->at || !k_new->at || !v_new->at || !out->at || !block_table || !ctx_len)
    return fail(SPEC_EINVAL, "a required pointer is NULL");
  spec_status_t s = check_attention_shape(batch, M, q_heads, kv_heads, head_dim, dtype);
  if (s != SPEC_OK) return s;
  if (M > 0 && !node_parent) return fail(SPEC_EINVAL, "node_parent is NULL");
  const int esz = element_bytes(dtype);
  if (max_blocks < 1) return fail(SPEC_EINVAL, "max_blocks must be >= 1");
  if ((int64_t)max_blocks * block_size > kMaxSlots) return fail(SPEC_ESHAPE, "max_blocks * block_size exceeds 2^30");
  if (k_new->seq_stride != v_new->seq_stride || k_new->row_stride != v_new->row_stride || k_new->head_stride != v_new->head_stride)
    return fail(SPEC_ESHAPE, "k_new and v_new must have the same strides");
  if (!rows_aligned(*q, esz) || !rows_aligned(*k_new, esz) || !rows_aligned(*v_new, esz) || !rows_aligned(*out, esz))
    return fail(SPEC_EINVAL, "rows of q, k_new, v_new and out must start on multiples of 16 bytes");
  const int64_t need = attention_workspace(batch, M, q_heads, kv_heads, head_dim, dtype == SPEC_BF16);
  if (need > 0 && (!workspace || workspace_bytes < need))
    return fail(SPEC_EINVAL, "workspace of %lld bytes, needed are %lld", (long long)(workspace ? workspace_bytes : 0), (long long)need);
  if (reinterpret_cast<uintptr_t>(workspace) & 15) return fail(SPEC_EINVAL, "workspace must be 16-byte aligned");
  return SPEC_OK;
}
static AttentionJob attention_job(const spec_rows_t& q, const spec_rows_t& k_new, const spec_rows_t& v_new, const spec_rows_t& out,
                                  const int32_t* block_table, const int32_t* ctx_len, const int32_t* node_parent, const int32_t* n_nodes,
                                  int32_t batch, int32_t M, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int esz, int32_t max_blocks,
                                  float scale, void* workspace) {
  AttentionJob j = {};
  j.q = q.at, j.k_new = k_new.at, j.v_new = v_new.at, j.out = const_cast<void*>(out.at);
  j.q_seq = q.seq_stride * esz, j.q_row = q.row_stride * esz, j.q_head = q.head_stride * esz;
  j.new_seq = k_new.seq_stride * esz, j.new_row = k_new.row_stride * esz, j.new_head = k_new.head_stride * esz;
  j.out_seq = out.seq_stride * esz, j.out_row = out.row_stride * esz, j.out_head = out.head_stride * esz;
  j.block_table = block_table, j.ctx_len = ctx_len, j.node_parent = node_parent, j.n_nodes = n_nodes;
  j.batch = batch, j.M = M, j.q_heads = q_heads, j.kv_heads = kv_heads, j.head_dim = head_dim;
  j.max_blocks = max_blocks, j.scale = scale, j.workspace = workspace;
  return j;
}
// (strides of 2^31 and more do not multiply beyond 63 bits: a tensor's bytes are addressable)
static int64_t offsets_most(const AttentionJob& j, int esz) { return (1ll << 32) - 64 - j.head_dim * esz; }
static bool rows_fit(const AttentionJob& j, int esz) { return j.new_row >= 0 && j.new_row * j.M <= offsets_most(j, esz); }

extern "C" spec_status_t spec_tree_attention(const spec_rows_t* q, const spec_rows_t* k_new, const spec_rows_t* v_new,
                                             const spec_cache_t* cache, const int32_t* block_table, const int32_t* ctx_len,
                                             const int32_t* node_parent, const int32_t* n_nodes, const spec_rows_t* out,
                                             int32_t batch, int32_t M, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                                             int32_t dtype, int32_t max_blocks, float scale, void* workspace,
                                             int64_t workspace_bytes, void* hip_stream) {
  if (!cache) return fail(SPEC_EINVAL, "a required pointer is NULL");
  spec_status_t s = check_attention(q, k_new, v_new, block_table, ctx_len, node_parent, out, batch, M, q_heads, kv_heads, head_dim, dtype, cache->block_size,
                                    max_blocks, workspace, workspace_bytes);
  if (s != SPEC_OK) return s;
  const int esz = element_bytes(dtype);
  s = check_cache(*cache, esz);
  if (s != SPEC_OK) return s;
  if (!rows_apart({{batch, out->seq_stride}, {M + 1, out->row_stride}, {q_heads, out->head_stride}}, head_dim))
    return fail(SPEC_EINVAL, "rows of out overlap");
  AttentionJob j = attention_job(*q, *k_new, *v_new, *out, block_table, ctx_len, node_parent, n_nodes, batch, M, q_heads, kv_heads, head_dim, esz, max_blocks, scale, workspace);
  j.k = cache->k, j.v = cache->v;
  j.block = cache->block_stride * esz, j.slot = cache->slot_stride * esz, j.cache_head = cache->head_stride * esz;
  j.n_blocks = cache->n_blocks, j.block_size = cache->block_size;
  j.one_place = cache->block_size % 16 == 0 && j.slot >= 0 && j.slot < (1 << 26);
  j.offsets_fit = rows_fit(j, esz) && j.block >= 0 && j.slot >= 0 &&
                  j.block * (cache->n_blocks - 1) + j.slot * (cache->block_size - 1) <= offsets_most(j, esz);
  HIP_TRY(launch_attention(j, dtype == SPEC_BF16, static_cast<hipStream_t>(hip_stream)));
  return SPEC_OK;
}

extern "C" spec_status_t spec_cache_extend(const int32_t* ctx_len, const int32_t* add, int32_t* new_len, int32_t* added,
                                           int32_t batch, int32_t* block_table, int32_t max_blocks, int32_t* ring,
                                           int32_t n_blocks, const int32_t* ring_state, int32_t* ring_state_new,
                                           int32_t block_size, int32_t* row_start, int32_t* slot, int32_t* pos,
                                           int32_t* src_row, int32_t cap, const int32_t* path_row, int32_t path_width,
                                           int32_t seq_rows, void* hip_stream) {
  if (!ctx_len || !add || !new_len || !added || !block_table || !ring || !ring_state || !ring_state_new || !row_start)
    return fail(SPEC_EINVAL, "a required pointer is NULL");
  if (batch < 1 || batch > 65535) return fail(SPEC_EINVAL, "batch = %d outside [1, 65535]", batch);
  if (max_blocks < 1 || n_blocks < 1 || block_size < 1) return fail(SPEC_EINVAL, "max_blocks, n_blocks and block_size must be >= 1");
  if (cap < 0 || (cap > 0 && !slot)) return fail(SPEC_EINVAL, "cap = %d, slot %s", cap, slot ? "given" : "NULL");
  if ((int64_t)n_blocks * block_size > kMaxSlots || (int64_t)max_blocks * block_size > kMaxSlots || cap > kMaxSlots)
    return fail(SPEC_ESHAPE, "n_blocks * block_size, max_blocks * block_size or cap exceeds 2^30");
  if (path_row) {
    if (cap > 0 && !src_row) return fail(SPEC_EINVAL, "src_row is NULL");
    if (path_width < 1 || seq_rows < 1) return fail(SPEC_EINVAL, "path_width and seq_rows must be >= 1");
    if ((int64_t)batch * seq_rows > 0x7fffffffLL) return fail(SPEC_ESHAPE, "batch * seq_rows is too large");
  }
  if (added == ctx_len || added == add || added == new_len || new_len == add || row_start == ctx_len || row_start == add)
    return fail(SPEC_EINVAL, "buffers overlap: only new_len may be ctx_len, and ring_state_new ring_state");
  const ExtendJob j = {ctx_len, add, new_len, added, batch, block_table, max_blocks, ring, n_blocks, ring_state, ring_state_new,
                       block_size, row_start, slot, pos, src_row, cap, path_row, path_width, seq_rows};
  HIP_TRY(launch_extend(j, static_cast<hipStream_t>(hip_stream)));
  return SPEC_OK;
}

extern "C" spec_status_t spec_cache_store(const spec_rows_t* k_new, const spec_rows_t* v_new, const spec_cache_t* cache,
                                          int64_t cache_layer_stride, int32_t layers, int32_t rows, int32_t kv_heads,
                                          int32_t head_dim, int32_t dtype, const int32_t* slot, const int32_t* src_row,
                                          int32_t count, void* hip_stream) {
  if (!k_new || !v_new || !cache) return fail(SPEC_EINVAL, "a required pointer is NULL");
  spec_status_t s = check_heads(dtype, kv_heads, head_dim);
  if (s != SPEC_OK) return s;
  if (layers < 1 || layers > 65535 || rows < 0 || count < 0)
    return fail(SPEC_EINVAL, "layers = %d outside [1, 65535], or rows = %d, count = %d negative", layers, rows, count);
  const int esz = element_bytes(dtype);
  s = check_cache(*cache, esz);
  if (s != SPEC_OK) return s;
  if (count == 0 || rows == 0) return SPEC_OK;
  if (!k_new->at || !v_new->at || !slot) return fail(SPEC_EINVAL, "a required pointer is NULL");
  if (k_new->seq_stride != v_new->seq_stride || k_new->row_stride != v_new->row_stride || k_new->head_stride != v_new->head_stride)
    return fail(SPEC_ESHAPE, "k_new and v_new must have the same strides");
  if (!rows_aligned(*k_new, esz) || !rows_aligned(*v_new, esz) || ((uint64_t)(cache_layer_stride * esz) & 15))
    return fail(SPEC_EINVAL, "rows of k_new, v_new and the cache must start on multiples of 16 bytes");
  if ((int64_t)kv_heads * head_dim > 1 << 24) return fail(SPEC_ESHAPE, "kv_heads * head_dim is too large");
  if (!rows_apart({{layers, cache_layer_stride}, {cache->n_blocks, cache->block_stride}, {cache->block_size, cache->slot_stride}, {kv_heads, cache->head_stride}}, head_dim))
    return fail(SPEC_EINVAL, "rows of the cache overlap");
  StoreJob j;
  j.k_new = static_cast<const uint8_t*>(k_new->at), j.v_new = static_cast<const uint8_t*>(v_new->at);
  j.k = static_cast<uint8_t*>(const_cast<void*>(cache->k)), j.v = static_cast<uint8_t*>(const_cast<void*>(cache->v));
  j.new_layer = k_new->seq_stride * esz, j.new_row = k_new->row_stride * esz, j.new_head = k_new->head_stride * esz;
  j.layer = cache_layer_stride * esz, j.block = cache->block_stride * esz, j.slot_stride = cache->slot_stride * esz;
  j.head = cache->head_stride * esz;
  j.layers = layers, j.rows = rows, j.kv_heads = kv_heads, j.row_words = head_dim * esz / 16;
  j.n_slots = cache->n_blocks * cache->block_size, j.block_size = cache->block_size;
  j.slot = slot, j.src_row = src_row, j.count = count;
  HIP_TRY(launch_store(j, static_cast<hipStream_t>(hip_stream)));
  return SPEC_OK;
}

// ---- rows of heads: norm and rotation, into a cache ---------------------------------------------------------------

// Rotation of heads of head_dim elements; pos: whether positions are given
static spec_status_t check_rotation(const spec_rotation_t* r, int32_t head_dim, int esz, bool pos) {
  if (!r) return SPEC_OK;
  if (!r->cos || !r->sin || !pos) return fail(SPEC_EINVAL, "a rotation needs cos, sin and positions");
  if (r->n_pos < 1) return fail(SPEC_EINVAL, "n_pos must be >= 1");
  if (r->pairs != 0 && r->pairs != 1) return fail(SPEC_EINVAL, "pairs = %d is neither 0 nor 1", r->pairs);
  const int per = 32 / esz;   // two words of 16 bytes
  if (r->rot_dim < per || r->rot_dim > head_dim || r->rot_dim % per)
    return fail(SPEC_ESHAPE, "rot_dim = %d must be a multiple of %d, at most head_dim = %d", r->rot_dim, per, head_dim);
  if ((reinterpret_cast<uintptr_t>(r->cos) | reinterpret_cast<uintptr_t>(r->sin)) & 15)
    return fail(SPEC_EINVAL, "cos and sin must be 16-byte aligned");
  return SPEC_OK;
}
static spec_status_t check_norm(const float* weight, double eps) {
  if (!weight) return SPEC_OK;
  if (reinterpret_cast<uintptr_t>(weight) & 15) return fail(SPEC_EINVAL, "weights of a norm must be 16-byte aligned");
  if (!(eps >= 0) || !(eps < 1e300)) return fail(SPEC_EINVAL, "eps = %g is negative or not finite", eps);
  return SPEC_OK;
}
template <typename Job>
static void set_rotation(Job& j, const spec_rotation_t* r, int esz) {
  j.cos = r ? r->cos : nullptr, j.sin = r ? r->sin : nullptr;
  j.n_pos = r ? r->n_pos : 0, j.half_words = r ? r->rot_dim * esz / 32 : 0, j.pairs = r ? r->pairs : 0;
}

extern "C" spec_status_t spec_rotate_rows(const spec_rows_t* q, const spec_rows_t* k, const spec_rows_t* q_out, const spec_rows_t* k_out,
                                          int32_t batch, int32_t M, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t dtype,
                                          const int32_t* pos, const int32_t* ctx_len, const int32_t* node_depth, const int32_t* n_nodes,
                                          const spec_rotation_t* rotation, const float* q_weight, const float* k_weight, double eps,
                                          void* hip_stream) {
  if (!q || !q_out || !q->at || !q_out->at || !k != !k_out || (k && (!k->at || !k_out->at)))
    return fail(SPEC_EINVAL, "a required pointer is NULL (k and k_out go together)");
  spec_status_t s = check_heads(dtype, k ? kv_heads : 1, head_dim);
  if (s != SPEC_OK) return s;
  if (batch < 1 || M < 0 || q_heads < 1) return fail(SPEC_EINVAL, "batch and q_heads must be >= 1, M >= 0");
  if (q_heads > 65535 || (k && kv_heads > 65535)) return fail(SPEC_ESHAPE, "q_heads = %d or kv_heads = %d exceeds 65535", q_heads, kv_heads);
  if ((int64_t)batch * ((int64_t)M + 1) > kMaxHeadEntries) return fail(SPEC_ESHAPE, "batch * (M + 1) exceeds %d", kMaxHeadEntries);
  if (pos && (ctx_len || node_depth)) return fail(SPEC_EINVAL, "positions are given by pos, or by ctx_len and node_depth");
  const int esz = element_bytes(dtype);
  s = check_rotation(rotation, head_dim, esz, pos || (ctx_len && (M == 0 || node_depth)));
  if (s == SPEC_OK) s = check_norm(q_weight, eps);
  if (s == SPEC_OK) s = check_norm(k_weight, eps);
  if (s != SPEC_OK) return s;
  if (k_weight && !k) return fail(SPEC_EINVAL, "k_weight without k");
  if (!rows_aligned(*q, esz) || !rows_aligned(*q_out, esz) || (k && (!rows_aligned(*k, esz) || !rows_aligned(*k_out, esz))))
    return fail(SPEC_EINVAL, "rows of q, k, q_out and k_out must start on multiples of 16 bytes");
  if (!rows_apart({{batch, q_out->seq_stride}, {M + 1, q_out->row_stride}, {q_heads, q_out->head_stride}}, head_dim) ||
      (k && !rows_apart({{batch, k_out->seq_stride}, {M + 1, k_out->row_stride}, {kv_heads, k_out->head_stride}}, head_dim)))
    return fail(SPEC_EINVAL, "rows of q_out or of k_out overlap");
  HeadsJob j = {};
  for (int i = 0; i < 2; ++i) {
    const spec_rows_t *from = i ? k : q, *to = i ? k_out : q_out;
    if (!from) continue;
    j.side[i] = {static_cast<const uint8_t*>(from->at), static_cast<uint8_t*>(const_cast<void*>(to->at)), from->seq_stride * esz, from->row_stride * esz,
                 from->head_stride * esz, to->seq_stride * esz, 0, to->row_stride * esz, to->head_stride * esz, i ? k_weight : q_weight,
                 i ? kv_heads : q_heads, true};
  }
  j.entries = batch * (M + 1), j.layers = 1, j.row_words = head_dim * esz / 16, j.head_dim = head_dim;
  set_rotation(j, rotation, esz);
  j.eps = eps, j.pos = pos, j.M = M, j.ctx_len = ctx_len, j.node_depth = node_depth, j.n_nodes = n_nodes;
  HIP_TRY(launch_heads(j, dtype == SPEC_BF16, false, static_cast<hipStream_t>(hip_stream)));
  return SPEC_OK;
}

// What spec_cache_append and spec_packed_append check alike; *work: whether there is anything to do
static spec_status_t check_append(const spec_rows_t* k_new, const spec_rows_t* v_new, int32_t layers, int32_t rows, int32_t kv_heads,
                                  int32_t head_dim, int32_t dtype, const int32_t* slot, const int32_t* pos, int32_t count,
                                  const spec_rotation_t* rotation, const float* k_weight, double eps, bool* work) {
  if (!k_new || !v_new) return fail(SPEC_EINVAL, "a required pointer is NULL");
  spec_status_t s = check_heads(dtype, kv_heads, head_dim);
  if (s != SPEC_OK) return s;
  if (layers < 1 || layers > 65535 || rows < 0 || count < 0)
    return fail(SPEC_EINVAL, "layers = %d outside [1, 65535], or rows = %d, count = %d negative", layers, rows, count);
  if (count > kMaxHeadEntries || kv_heads > 65535) return fail(SPEC_ESHAPE, "count = %d exceeds %d, or kv_heads = %d 65535", count, kMaxHeadEntries, kv_heads);
  const int esz = element_bytes(dtype);
  *work = count > 0 && rows > 0;
  if (*work && (!k_new->at || !v_new->at || !slot)) return fail(SPEC_EINVAL, "a required pointer is NULL");
  s = check_rotation(rotation, head_dim, esz, pos || !*work);
  if (s == SPEC_OK) s = check_norm(k_weight, eps);
  if (s != SPEC_OK) return s;
  if (k_new->seq_stride != v_new->seq_stride || k_new->row_stride != v_new->row_stride || k_new->head_stride != v_new->head_stride)
    return fail(SPEC_ESHAPE, "k_new and v_new must have the same strides");
  if (*work && (!rows_aligned(*k_new, esz) || !rows_aligned(*v_new, esz)))
    return fail(SPEC_EINVAL, "rows of k_new and v_new must start on multiples of 16 bytes");
  return SPEC_OK;
}

extern "C" spec_status_t spec_cache_append(const spec_rows_t* k_new, const spec_rows_t* v_new, const spec_cache_t* cache,
                                           int64_t cache_layer_stride, int32_t layers, int32_t rows, int32_t kv_heads, int32_t head_dim,
                                           int32_t dtype, const int32_t* slot, const int32_t* src_row, const int32_t* pos, int32_t count,
                                           const spec_rotation_t* rotation, const float* k_weight, double eps, void* hip_stream) {
  if (!cache) return fail(SPEC_EINVAL, "a required pointer is NULL");
  bool work = false;
  spec_status_t s = check_append(k_new, v_new, layers, rows, kv_heads, head_dim, dtype, slot, pos, count, rotation, k_weight, eps, &work);
  if (s != SPEC_OK) return s;
  const int esz = element_bytes(dtype);
  s = check_cache(*cache, esz);
  if (s != SPEC_OK) return s;
  if ((uint64_t)(cache_layer_stride * esz) & 15) return fail(SPEC_EINVAL, "rows of the cache must start on multiples of 16 bytes");
  if (!rows_apart({{layers, cache_layer_stride}, {cache->n_blocks, cache->block_stride}, {cache->block_size, cache->slot_stride}, {kv_heads, cache->head_stride}}, head_dim))
    return fail(SPEC_EINVAL, "rows of the cache overlap");
  if (!work) return SPEC_OK;
  HeadsJob j = {};
  for (int i = 0; i < 2; ++i) {
    const spec_rows_t& from = i ? *v_new : *k_new;
    j.side[i] = {static_cast<const uint8_t*>(from.at), static_cast<uint8_t*>(const_cast<void*>(i ? cache->v : cache->k)), from.seq_stride * esz,
                 from.row_stride * esz, from.head_stride * esz, cache_layer_stride * esz, cache->block_stride * esz, cache->slot_stride * esz,
                 cache->head_stride * esz, i ? nullptr : k_weight, kv_heads, i == 0};
  }
  j.entries = count, j.layers = layers, j.row_words = head_dim * esz / 16, j.head_dim = head_dim;
  set_rotation(j, rotation, esz);
  j.eps = eps, j.pos = pos, j.slot = slot, j.src_row = src_row, j.rows = rows;
  j.n_slots = cache->n_blocks * cache->block_size, j.block_size = cache->block_size;
  HIP_TRY(launch_heads(j, dtype == SPEC_BF16, true, static_cast<hipStream_t>(hip_stream)));
  return SPEC_OK;
}

// A cache of four bits: rows of head_dim / 2 bytes of codes and head_dim / 32 of scales
static spec_status_t check_packed(const spec_packed_t* c, int32_t head_dim) {
  if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return fail(SPEC_EINVAL, "the cache, or its codes or scales, is NULL");
  if (head_dim < 32 || head_dim % 32 || head_dim > 256) return fail(SPEC_ESHAPE, "head_dim = %d must be a multiple of 32, at most 256", head_dim);
  if (c->n_blocks < 1 || c->block_size < 1) return fail(SPEC_EINVAL, "n_blocks and block_size must be >= 1");
  if ((int64_t)c->n_blocks * c->block_size > kMaxSlots) return fail(SPEC_ESHAPE, "n_blocks * block_size exceeds 2^30");
  if (!rows_aligned(c->k, c->block_stride, c->slot_stride, c->head_stride, 1) || (reinterpret_cast<uintptr_t>(c->v) & 15))
    return fail(SPEC_EINVAL, "rows of codes must start on multiples of 16 bytes");
  return SPEC_OK;
}

extern "C" spec_status_t spec_packed_append(const spec_rows_t* k_new, const spec_rows_t* v_new, const spec_packed_t* cache,
                                            int64_t cache_layer_stride, int64_t scale_layer_stride, int32_t layers, int32_t rows,
                                            int32_t kv_heads, int32_t head_dim, const int32_t* slot, const int32_t* src_row,
                                            const int32_t* pos, int32_t count, const spec_rotation_t* rotation, const float* k_weight,
                                            double eps, void* hip_stream) {
  spec_status_t s = check_packed(cache, head_dim);
  if (s != SPEC_OK) return s;
  bool work = false;
  s = check_append(k_new, v_new, layers, rows, kv_heads, head_dim, SPEC_BF16, slot, pos, count, rotation, k_weight, eps, &work);
  if (s != SPEC_OK) return s;
  if (cache_layer_stride & 15) return fail(SPEC_EINVAL, "rows of codes must start on multiples of 16 bytes");
  if (!rows_apart({{layers, cache_layer_stride}, {cache->n_blocks, cache->block_stride}, {cache->block_size, cache->slot_stride}, {kv_heads, cache->head_stride}}, head_dim / 2) ||
      !rows_apart({{layers, scale_layer_stride}, {cache->n_blocks, cache->scale_block_stride}, {cache->block_size, cache->scale_slot_stride}, {kv_heads, cache->scale_head_stride}}, head_dim / 32))
    return fail(SPEC_EINVAL, "rows of the cache overlap");
  if (!work) return SPEC_OK;
  PackJob j = {};
  j.k_new = static_cast<const uint8_t*>(k_new->at), j.v_new = static_cast<const uint8_t*>(v_new->at);
  j.k = static_cast<uint8_t*>(const_cast<void*>(cache->k)), j.v = static_cast<uint8_t*>(const_cast<void*>(cache->v));
  j.k_scale = const_cast<uint8_t*>(cache->k_scale), j.v_scale = const_cast<uint8_t*>(cache->v_scale);
  j.new_layer = k_new->seq_stride * 2, j.new_row = k_new->row_stride * 2, j.new_head = k_new->head_stride * 2;
  j.layer = cache_layer_stride, j.block = cache->block_stride, j.slot_stride = cache->slot_stride, j.head = cache->head_stride;
  j.scale_layer = scale_layer_stride, j.scale_block = cache->scale_block_stride, j.scale_slot = cache->scale_slot_stride, j.scale_head = cache->scale_head_stride;
  j.entries = count, j.layers = layers, j.rows = rows, j.heads = kv_heads, j.groups = head_dim / 32;
  set_rotation(j, rotation, 2);
  j.weight = k_weight, j.eps = eps, j.pos = pos, j.slot = slot, j.src_row = src_row;
  j.n_slots = cache->n_blocks * cache->block_size, j.block_size = cache->block_size;
  HIP_TRY(launch_pack(j, static_cast<hipStream_t>(hip_stream)));
  return SPEC_OK;
}

extern "C" spec_status_t spec_packed_load(const spec_packed_t* cache, int64_t cache_layer_stride, int64_t scale_layer_stride, int32_t layers,
                                          int32_t kv_heads, int32_t head_dim, const int32_t* slot, int32_t count, const spec_rows_t* k_out,
                                          const spec_rows_t* v_out, void* hip_stream) {
  spec_status_t s = check_packed(cache, head_dim);
  if (s == SPEC_OK) s = check_heads(SPEC_BF16, kv_heads, head_dim);
  if (s != SPEC_OK) return s;
  if (!k_out || !v_out) return fail(SPEC_EINVAL, "a required pointer is NULL");
  if (layers < 1 || layers > 65535 || count < 0) return fail(SPEC_EINVAL, "layers = %d outside [1, 65535], or count = %d negative", layers, count);
  if (cache_layer_stride & 15) return fail(SPEC_EINVAL, "rows of codes must start on multiples of 16 bytes");
  if (kv_heads > 65535) return fail(SPEC_ESHAPE, "kv_heads = %d exceeds 65535", kv_heads);
  if (count == 0) return SPEC_OK;
  if (!slot || !k_out->at || !v_out->at) return fail(SPEC_EINVAL, "a required pointer is NULL");
  if (k_out->seq_stride != v_out->seq_stride || k_out->row_stride != v_out->row_stride || k_out->head_stride != v_out->head_stride)
    return fail(SPEC_ESHAPE, "k_out and v_out must have the same strides");
  if (!rows_aligned(*k_out, 2) || !rows_aligned(*v_out, 2)) return fail(SPEC_EINVAL, "rows of k_out and v_out must start on multiples of 16 bytes");
  if (!rows_apart({{layers, k_out->seq_stride}, {count, k_out->row_stride}, {kv_heads, k_out->head_stride}}, head_dim))
    return fail(SPEC_EINVAL, "rows of k_out, or of v_out, overlap");
  UnpackJob j = {};
  j.k = static_cast<const uint8_t*>(cache->k), j.v = static_cast<const uint8_t*>(cache->v), j.k_scale = cache->k_scale, j.v_scale = cache->v_scale;
  j.k_out = static_cast<uint8_t*>(const_cast<void*>(k_out->at)), j.v_out = static_cast<uint8_t*>(const_cast<void*>(v_out->at));
  j.layer = cache_layer_stride, j.block = cache->block_stride, j.slot_stride = cache->slot_stride, j.head = cache->head_stride;
  j.scale_layer = scale_layer_stride, j.scale_block = cache->scale_block_stride, j.scale_slot = cache->scale_slot_stride, j.scale_head = cache->scale_head_stride;
  j.out_layer = k_out->seq_stride * 2, j.out_row = k_out->row_stride * 2, j.out_head = k_out->head_stride * 2;
  j.count = count, j.layers = layers, j.heads = kv_heads, j.groups = head_dim / 32, j.slot = slot;
  j.n_slots = cache->n_blocks * cache->block_size, j.block_size = cache->block_size;
  HIP_TRY(launch_unpack(j, static_cast<hipStream_t>(hip_stream)));
  return SPEC_OK;
}

extern "C" spec_status_t spec_packed_attention_workspace(int32_t batch, int32_t M, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                                                         int64_t* bytes) {
  if (!bytes) return fail(SPEC_EINVAL, "bytes is NULL");
  spec_status_t s = check_attention_shape(batch, M, q_heads, kv_heads, head_dim, SPEC_BF16);
  if (s != SPEC_OK) return s;
  if (head_dim % 32) return fail(SPEC_ESHAPE, "head_dim = %d must be a multiple of 32", head_dim);
  *bytes = attention_workspace(batch, M, q_heads, kv_heads, head_dim, true);
  return SPEC_OK;
}

extern "C" spec_status_t spec_packed_attention(const spec_rows_t* q, const spec_rows_t* k_new, const spec_rows_t* v_new,
                                               const spec_packed_t* cache, const int32_t* block_table, const int32_t* ctx_len,
                                               const int32_t* node_parent, const int32_t* n_nodes, const spec_rows_t* out,
                                               int32_t batch, int32_t M, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                                               int32_t max_blocks, float scale, void* workspace, int64_t workspace_bytes,
                                               void* hip_stream) {
  spec_status_t s = check_packed(cache, head_dim);
  if (s != SPEC_OK) return s;
  s = check_attention(q, k_new, v_new, block_table, ctx_len, node_parent, out, batch, M, q_heads, kv_heads, head_dim, SPEC_BF16, cache->block_size,
                      max_blocks, workspace, workspace_bytes);
  if (s != SPEC_OK) return s;
  if (!rows_apart({{batch, out->seq_stride}, {M + 1, out->row_stride}, {q_heads, out->head_stride}}, head_dim))
    return fail(SPEC_EINVAL, "rows of out overlap");
  AttentionJob j = attention_job(*q, *k_new, *v_new, *out, block_table, ctx_len, node_parent, n_nodes, batch, M, q_heads, kv_heads, head_dim, 2, max_blocks, scale, workspace);
  j.k = cache->k, j.v = cache->v, j.k_scale = cache->k_scale, j.v_scale = cache->v_scale;
  j.block = cache->block_stride, j.slot = cache->slot_stride, j.cache_head = cache->head_stride;
  j.scale_block = cache->scale_block_stride, j.scale_slot = cache->scale_slot_stride, j.scale_head = cache->scale_head_stride;
  j.n_blocks = cache->n_blocks, j.block_size = cache->block_size;
  j.one_place = cache->block_size % 16 == 0 && j.slot >= 0 && j.slot < (1 << 26) && j.scale_slot >= 0 && j.scale_slot < (1 << 26);
  j.offsets_fit = rows_fit(j, 2);
  HIP_TRY(launch_packed_attention(j, static_cast<hipStream_t>(hip_stream)));
  return SPEC_OK;
}

static spec_status_t check_logits(const void* logits, int32_t dtype, int32_t batch, int32_t M, int32_t vocab,
                                  const spec_penalties_t* pen, const int32_t* node_tok, const int32_t* node_parent) {
  if (!logits) return fail(SPEC_EINVAL, "logits is NULL");
  if (!known_dtype(dtype)) return fail(SPEC_EDTYPE, "logits_dtype = %d is neither SPEC_F32 nor SPEC_BF16", dtype);
  if (batch < 1 || M < 0 || vocab < 1) return fail(SPEC_EINVAL, "batch and vocab must be >= 1, M >= 0");
  if (M > kMaxTreeItems) return fail(SPEC_ESHAPE, "M = %d exceeds %d", M, kMaxTreeItems);
  // (a launch has fewer than 2^32 threads, and a row up to 512 of them in so many rows)
  if ((int64_t)batch * (M + 1) > kMaxLogitsRows) return fail(SPEC_ESHAPE, "batch * (M + 1) = %lld exceeds %d", (long long)batch * (M + 1), kMaxLogitsRows);
  if (vocab > 1 << 30) return fail(SPEC_ESHAPE, "vocab exceeds 2^30");
  if (!node_tok != !node_parent) return fail(SPEC_EINVAL, "node_tok and node_parent go together");
  if (pen) {
    if (pen->bias && (!pen->bias_row || pen->n_bias < 0)) return fail(SPEC_EINVAL, "bias needs bias_row and n_bias >= 0");
    if (pen->allowed && (!pen->mask_row || pen->n_allowed < 0)) return fail(SPEC_EINVAL, "allowed needs mask_row and n_allowed >= 0");
  }
  return SPEC_OK;
}

extern "C" spec_status_t spec_penalize(const void* logits, int32_t logits_dtype, int32_t batch, int32_t M, int32_t vocab,
                                       const spec_penalties_t* pen, const int32_t* node_tok, const int32_t* node_parent,
                                       const int32_t* n_nodes, void* out, void* hip_stream) {
  spec_status_t s = check_logits(logits, logits_dtype, batch, M, vocab, pen, node_tok, node_parent);
  if (s != SPEC_OK) return s;
  if (!pen || !out) return fail(SPEC_EINVAL, "a required pointer is NULL");
  const LogitsJob j = {logits, batch, M, vocab, *pen, M > 0 ? node_tok : nullptr, node_parent, n_nodes, out, nullptr};
  HIP_TRY(launch_logits(j, logits_dtype == SPEC_BF16, static_cast<hipStream_t>(hip_stream)));
  return SPEC_OK;
}

extern "C" spec_status_t spec_verify_tree(const void* logits, int32_t logits_dtype, const int32_t* cand_tokens,
                                          const int32_t* cand_node, const int32_t* n_cand, const int32_t* node_tok,
                                          const int32_t* node_parent, const int32_t* n_nodes, const spec_penalties_t* pen,
                                          int32_t batch, int32_t M, int32_t B, int32_t n_predict, int32_t vocab,
                                          int32_t* greedy, int32_t* accept_len, int32_t* best_cand, int32_t* out_tokens,
                                          int32_t* n_out, int32_t* path_row, int32_t* accept_all, int32_t* counts_out,
                                          uint32_t* seen_out, void* hip_stream) {
  spec_status_t s = check_logits(logits, logits_dtype, batch, M, vocab, pen, node_tok, node_parent);
  if (s != SPEC_OK) return s;
  if (!greedy || !accept_len || !best_cand || !out_tokens || !n_out || !path_row)
    return fail(SPEC_EINVAL, "a required pointer is NULL");
  if (B < 1 || n_predict < 0 || n_predict > SPEC_MAX_STAGES)
    return fail(SPEC_EINVAL, "B = %d must be >= 1, n_predict = %d within [0, %d]", B, n_predict, SPEC_MAX_STAGES);
  if ((int64_t)B * n_predict > kMaxTreeItems) return fail(SPEC_ESHAPE, "B * n_predict = %lld exceeds %d", (long long)B * n_predict, kMaxTreeItems);
  if (n_predict == 0 && B != 1) return fail(SPEC_ESHAPE, "n_predict = 0 needs B = 1");
  if (n_predict > 0 && (!cand_tokens || !cand_node)) return fail(SPEC_EINVAL, "cand_tokens or cand_node is NULL");
  spec_penalties_t none = {};
  const LogitsJob j = {logits, batch, M, vocab, pen ? *pen : none, M > 0 && pen ? node_tok : nullptr, node_parent, n_nodes,
                       nullptr, greedy};
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  HIP_TRY(launch_logits(j, logits_dtype == SPEC_BF16, st));
  const AcceptTreeJob a = {greedy, cand_tokens, cand_node, n_cand, n_nodes, batch, M, B, n_predict, vocab, accept_len, best_cand,
                           out_tokens, n_out, path_row, accept_all, counts_out, seen_out};
  HIP_TRY(launch_accept_tree(a, st));
  return SPEC_OK;
}

static spec_status_t check_sampled(int32_t batch, int32_t M, int32_t vocab) {
  // (a launch has fewer than 2^32 threads: 256 for each of up to 64 parts of a row of every sequence, or of the parts of few rows)
  if (batch > kMaxSampledBatch || (int64_t)batch * (M + 1) > kMaxSampledRows)
    return fail(SPEC_ESHAPE, "batch = %d exceeds %d, or batch * (M + 1) = %lld %d", batch, kMaxSampledBatch, (long long)batch * (M + 1), kMaxSampledRows);
  return vocab > 1 << 30 ? fail(SPEC_ESHAPE, "vocab exceeds 2^30") : SPEC_OK;
}

extern "C" spec_status_t spec_verify_sampled_workspace(int32_t batch, int32_t M, int32_t vocab, int32_t logits_dtype, int64_t* bytes) {
  if (!bytes) return fail(SPEC_EINVAL, "bytes is NULL");
  if (!known_dtype(logits_dtype)) return fail(SPEC_EDTYPE, "logits_dtype = %d is neither SPEC_F32 nor SPEC_BF16", logits_dtype);
  if (batch < 1 || M < 0 || vocab < 1) return fail(SPEC_EINVAL, "batch and vocab must be >= 1, M >= 0");
  if (M > kMaxTreeItems) return fail(SPEC_ESHAPE, "M = %d exceeds %d", M, kMaxTreeItems);
  spec_status_t s = check_sampled(batch, M, vocab);
  if (s != SPEC_OK) return s;
  *bytes = sample_workspace(batch, M, vocab);
  return SPEC_OK;
}

extern "C" spec_status_t spec_verify_sampled(const void* logits, int32_t logits_dtype, const int32_t* node_tok, const int32_t* node_parent,
                                             const int32_t* n_nodes, const spec_penalties_t* pen, const float* temperature,
                                             const float* uniform, int32_t batch, int32_t M, int32_t n_predict, int32_t vocab,
                                             int32_t* accept_len, int32_t* out_tokens, int32_t* n_out, int32_t* path_row, float* out_logp,
                                             int32_t* counts_out, uint32_t* seen_out, void* workspace, int64_t workspace_bytes,
                                             void* hip_stream) {
  spec_status_t s = check_logits(logits, logits_dtype, batch, M, vocab, pen, node_tok, node_parent);
  if (s == SPEC_OK) s = check_sampled(batch, M, vocab);
  if (s != SPEC_OK) return s;
  if (!uniform || !accept_len || !out_tokens || !n_out || !path_row) return fail(SPEC_EINVAL, "a required pointer is NULL");
  if (M > 0 && (!node_tok || !node_parent)) return fail(SPEC_EINVAL, "node_tok or node_parent is NULL");
  if (n_predict < 0 || n_predict > SPEC_MAX_STAGES) return fail(SPEC_EINVAL, "n_predict = %d outside [0, %d]", n_predict, SPEC_MAX_STAGES);
  const int64_t need = sample_workspace(batch, M, vocab);
  if (!workspace || workspace_bytes < need)
    return fail(SPEC_EINVAL, "workspace of %lld bytes, needed are %lld", (long long)(workspace ? workspace_bytes : 0), (long long)need);
  if (reinterpret_cast<uintptr_t>(workspace) & 15) return fail(SPEC_EINVAL, "workspace must be 16-byte aligned");
  spec_penalties_t none = {};
  SampleJob j = {};
  j.logits = logits, j.batch = batch, j.M = M, j.V = vocab, j.n = n_predict, j.pen = pen ? *pen : none, j.paths = pen != nullptr;
  j.node_tok = node_tok, j.node_parent = node_parent, j.n_nodes = n_nodes, j.temperature = temperature, j.uniform = uniform;
  j.accept_len = accept_len, j.out_tokens = out_tokens, j.n_out = n_out, j.path_row = path_row, j.out_logp = out_logp;
  j.counts = counts_out, j.seen = seen_out;
  HIP_TRY(launch_sample(j, workspace, logits_dtype == SPEC_BF16, static_cast<hipStream_t>(hip_stream)));
  return SPEC_OK;
}
