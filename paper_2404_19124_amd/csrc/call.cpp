// The binding's usual case in one native call: every tensor argument is checked (exact torch.Tensor, element type, shape,
// contiguous, on the device) and the library called with their addresses.  None is returned, and nothing has happened,
// where an argument is not of that kind: the binding then goes through its checks one by one and says what is wrong.
// Host only.  A verify and a hand-over check 18 tensors; in Python that was two thirds of the 18 us that both calls took,
// whose three kernels take 8: 18.5 -> 11.3 us back to back (32000 logits, 16 candidates of 3), 48 -> 34 for a first call.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <c10/core/impl/VirtualGuardImpl.h>
#include <torch/csrc/Device.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <iterator>

#include "../../include/spec.h"

namespace {

decltype(&spec_verify) f_verify;
decltype(&spec_verify_dynamic) f_verify_dynamic;
decltype(&spec_advance) f_advance;
decltype(&spec_tree_metadata) f_tree_metadata;
decltype(&spec_draft) f_draft;
decltype(&spec_tree_attention) f_tree_attention;
decltype(&spec_cache_extend) f_cache_extend;
decltype(&spec_cache_store) f_cache_store;
decltype(&spec_penalize) f_penalize;
decltype(&spec_verify_tree) f_verify_tree;
PyObject* f_stream;   // the binding's _stream_ptr

const at::Tensor* tensor(PyObject* o) { return THPVariable_CheckExact(o) ? &THPVariable_Unpack(o) : nullptr; }

template <typename T>
bool usual(PyObject* o, at::ScalarType dtype, std::initializer_list<int64_t> shape, T** at) {
  const at::Tensor* t = tensor(o);
  if (!t || t->scalar_type() != dtype || t->sizes() != at::IntArrayRef(shape) || !t->is_contiguous() || !t->is_cuda()) return false;
  *at = static_cast<T*>(t->mutable_data_ptr());
  return true;
}
template <typename T>
bool usual_or_none(PyObject* o, at::ScalarType dtype, std::initializer_list<int64_t> shape, T** at) {
  *at = nullptr;
  return o == Py_None || usual(o, dtype, shape, at);
}

// 4-dimensional float32 or bfloat16 input; false: not of that kind
bool floats4(PyObject* o, int64_t (&size)[4], int32_t* code, at::ScalarType* dtype, void** at) {
  const at::Tensor* t = tensor(o);
  if (!t || t->dim() != 4) return false;
  *dtype = t->scalar_type();
  if (*dtype == at::kFloat) *code = SPEC_F32;
  else if (*dtype == at::kBFloat16) *code = SPEC_BF16;
  else return false;
  for (int i = 0; i < 4; ++i) size[i] = t->size(i);
  for (int i = 0; i < 4; ++i)
    if (size[i] > INT32_MAX) return false;
  return usual(o, *dtype, {size[0], size[1], size[2], size[3]}, at);
}

// false with an exception set: the caller returns nullptr
bool stream_of(PyObject* o, void** stream) {
  PyObject* p = PyObject_CallOneArg(f_stream, o);
  if (!p) return false;
  *stream = p == Py_None ? nullptr : PyLong_AsVoidPtr(p);
  Py_DECREF(p);
  return !PyErr_Occurred();
}

template <typename F>
PyObject* status_of(F&& call) {
  spec_status_t s;
  Py_BEGIN_ALLOW_THREADS
  s = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(s);
}

// logits, cand_tokens, n_cand (None: spec_verify), greedy, accept_len, best_cand, out_tokens, n_out, accept_all, stream
PyObject* verify(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 10) Py_RETURN_NONE;
  try {
    int64_t d[4];
    int32_t code;
    at::ScalarType dt;
    void *logits, *stream;
    int32_t *cand, *n_cand, *greedy, *len, *best, *out, *n_out, *all;
    if (!floats4(a[0], d, &code, &dt, &logits)) Py_RETURN_NONE;
    const int64_t b = d[0], B = d[1], n1 = d[2];
    if (!usual(a[1], at::kInt, {b, B, n1 - 1}, &cand) || !usual_or_none(a[2], at::kInt, {b}, &n_cand) ||
        !usual(a[3], at::kInt, {b, B, n1}, &greedy) || !usual(a[4], at::kInt, {b}, &len) || !usual(a[5], at::kInt, {b}, &best) ||
        !usual(a[6], at::kInt, {b, n1}, &out) || !usual(a[7], at::kInt, {b}, &n_out) ||
        !usual_or_none(a[8], at::kInt, {b, B}, &all))
      Py_RETURN_NONE;
    if (!stream_of(a[9], &stream)) return nullptr;
    const int32_t V = (int32_t)d[3], np = (int32_t)n1 - 1;
    return status_of([&] {
      return n_cand ? f_verify_dynamic(logits, code, cand, n_cand, (int32_t)b, (int32_t)B, np, V, greedy, len, best, out, n_out, all, stream)
                    : f_verify(logits, code, cand, (int32_t)b, (int32_t)B, np, V, greedy, len, best, out, n_out, all, stream);
    });
  } catch (...) {   // a tensor without storage, say
    Py_RETURN_NONE;
  }
}

// hidden, best_cand, accept_len, out_tokens, next_state, next_tok, stream
PyObject* advance(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7) Py_RETURN_NONE;
  try {
    int64_t d[4];
    int32_t code;
    at::ScalarType dt;
    void *hidden, *state, *stream;
    int32_t *best, *len, *out, *tok;
    if (!floats4(a[0], d, &code, &dt, &hidden) || !usual(a[1], at::kInt, {d[0]}, &best) || !usual(a[2], at::kInt, {d[0]}, &len) ||
        !usual(a[3], at::kInt, {d[0], d[2]}, &out) || !usual(a[4], dt, {d[0], d[3]}, &state) || !usual(a[5], at::kInt, {d[0]}, &tok))
      Py_RETURN_NONE;
    if (!stream_of(a[6], &stream)) return nullptr;
    return status_of([&] {
      return f_advance(hidden, code, (int32_t)d[0], (int32_t)d[1], (int32_t)d[2] - 1, (int32_t)d[3], best, len, out, state, tok, stream);
    });
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// cand_tokens, node_tok, node_parent, node_depth, n_nodes, cand_node, mask, stream
PyObject* tree_metadata(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 8) Py_RETURN_NONE;
  try {
    const at::Tensor* t = tensor(a[0]);
    if (!t || t->dim() != 3) Py_RETURN_NONE;
    const int64_t b = t->size(0), B = t->size(1), np = t->size(2);
    if (b > INT32_MAX || B > INT32_MAX || np > INT32_MAX) Py_RETURN_NONE;
    const int64_t M = B * np;
    int32_t *cand, *tok, *parent, *depth, *count, *node;
    uint8_t* mask;
    void* stream;
    if (!usual(a[0], at::kInt, {b, B, np}, &cand) || !usual(a[1], at::kInt, {b, M}, &tok) || !usual(a[2], at::kInt, {b, M}, &parent) ||
        !usual(a[3], at::kInt, {b, M}, &depth) || !usual(a[4], at::kInt, {b}, &count) || !usual(a[5], at::kInt, {b, B, np}, &node) ||
        !usual_or_none(a[6], at::kByte, {b, M, M}, &mask))
      Py_RETURN_NONE;
    if (!stream_of(a[7], &stream)) return nullptr;
    return status_of([&] {
      return f_tree_metadata(cand, (int32_t)b, (int32_t)B, (int32_t)np, tok, parent, depth, count, node, mask, stream);
    });
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// handle (address or None), n_predict, emb_dim, weight_dtype, state, last_tok, top_k, B, cand_tokens, cand_scores, cand_leaf, stream
PyObject* draft(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 12 || !PyLong_CheckExact(a[0]) || !PyLong_CheckExact(a[7])) Py_RETURN_NONE;
  if (!PyTuple_CheckExact(a[6]) && !PyList_CheckExact(a[6])) Py_RETURN_NONE;
  try {
    const long np = PyLong_AsLong(a[1]), E = PyLong_AsLong(a[2]), code = PyLong_AsLong(a[3]);
    int over = 0;
    const long B = PyLong_AsLongAndOverflow(a[7], &over);
    if (over || B < 0 || B > INT32_MAX || np < 1 || np > SPEC_MAX_STAGES || (code != SPEC_F32 && code != SPEC_BF16) ||
        PySequence_Fast_GET_SIZE(a[6]) != np)
      Py_RETURN_NONE;
    int32_t top_k[SPEC_MAX_STAGES];
    for (long i = 0; i < np; ++i) {
      PyObject* k = PySequence_Fast_GET_ITEM(a[6], i);
      if (!PyLong_CheckExact(k)) Py_RETURN_NONE;
      const long v = PyLong_AsLongAndOverflow(k, &over);
      if (over || v < INT32_MIN || v > INT32_MAX) Py_RETURN_NONE;
      top_k[i] = (int32_t)v;
    }
    const at::Tensor* t = tensor(a[4]);
    if (!t || t->dim() != 2 || t->size(0) > INT32_MAX) Py_RETURN_NONE;
    const int64_t b = t->size(0);
    void *state, *stream;
    int32_t *last, *tokens, *leaf;
    float* scores;
    if (!usual(a[4], code == SPEC_BF16 ? at::kBFloat16 : at::kFloat, {b, E}, &state) || !usual(a[5], at::kInt, {b}, &last) ||
        !usual(a[8], at::kInt, {b, B, np}, &tokens) || !usual(a[9], at::kFloat, {b, B}, &scores) || !usual(a[10], at::kInt, {b, B}, &leaf))
      Py_RETURN_NONE;
    spec_model_t* model = static_cast<spec_model_t*>(PyLong_AsVoidPtr(a[0]));
    if (!stream_of(a[11], &stream)) return nullptr;
    return status_of([&] { return f_draft(model, state, last, (int32_t)b, top_k, (int32_t)B, tokens, scores, leaf, nullptr, stream); });
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// ---- the operators on the rows of a tree.  Their arguments lie on the current device, and so does the stream, for the kernels
// run there.  From Python's checks one by one: 24 us on the host for a verification, 17 for the others ----
struct Rows {
  int device = c10::impl::VirtualGuardImpl(c10::DeviceType::CUDA).getDevice().index();

  template <typename T>
  bool in(PyObject* o, at::ScalarType dtype, std::initializer_list<int64_t> shape, T** at) const {
    return usual(o, dtype, shape, at) && THPVariable_Unpack(o).get_device() == device;
  }
  template <typename T>
  bool maybe(PyObject* o, at::ScalarType dtype, std::initializer_list<int64_t> shape, T** at) const {
    *at = nullptr;
    return o == Py_None || in(o, dtype, shape, at);
  }
  // any strides but along the last dimension; 0 along dimensions of one entry, whose stride says nothing
  bool strided(PyObject* o, at::ScalarType dtype, std::initializer_list<int64_t> shape, int64_t* stride, void** at, bool written = false) const {
    const at::Tensor* t = tensor(o);
    if (!t || t->scalar_type() != dtype || t->sizes() != at::IntArrayRef(shape) || !t->is_cuda() || t->get_device() != device) return false;
    const int64_t last = t->dim() - 1;
    if (t->size(last) > 1 && t->stride(last) != 1) return false;
    for (int64_t i = 0; i < last; ++i) {
      stride[i] = t->size(i) > 1 ? t->stride(i) : 0;
      if (written && t->size(i) > 1 && stride[i] == 0) return false;
    }
    *at = t->mutable_data_ptr();
    return true;
  }
  // a stream of another device is the slow way's to refuse
  bool here(PyObject* stream) const {
    if (stream == Py_None) return true;
    PyObject* d = PyObject_GetAttrString(stream, "device");
    if (!d) {
      PyErr_Clear();
      return true;
    }
    const bool ok = !THPDevice_Check(d) || !reinterpret_cast<THPDevice*>(d)->device.has_index() ||
                    reinterpret_cast<THPDevice*>(d)->device.index() == device;
    Py_DECREF(d);
    return ok;
  }
};

// float32 or bfloat16 of `dim` dimensions, none over 2^31 - 1
bool floats(PyObject* o, int64_t dim, int64_t* size, int32_t* code, at::ScalarType* dtype) {
  const at::Tensor* t = tensor(o);
  if (!t || t->dim() != dim) return false;
  *dtype = t->scalar_type();
  if (*dtype == at::kFloat) *code = SPEC_F32;
  else if (*dtype == at::kBFloat16) *code = SPEC_BF16;
  else return false;
  for (int64_t i = 0; i < dim; ++i)
    if ((size[i] = t->size(i)) > INT32_MAX) return false;
  return true;
}

bool int32_of(PyObject* o, int32_t* x) {
  if (!PyLong_CheckExact(o)) return false;
  int over = 0;
  const long v = PyLong_AsLongAndOverflow(o, &over);
  if (over || v < INT32_MIN || v > INT32_MAX) return false;
  *x = (int32_t)v;
  return true;
}

// size of dimension `i` of a tensor of `dim` dimensions, -1: none
int64_t size_of(PyObject* o, int64_t dim, int64_t i) {
  const at::Tensor* t = tensor(o);
  return t && t->dim() == dim && t->size(i) <= INT32_MAX ? t->size(i) : -1;
}

// q, k_new, v_new, k_cache, v_cache, block_table, ctx_len, node_parent, n_nodes, out, workspace, scale (None or float), stream
PyObject* tree_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 13 || (a[11] != Py_None && !PyFloat_CheckExact(a[11]))) Py_RETURN_NONE;
  try {
    const Rows on;
    int64_t d[4], c[4], sv[3], cv[3];
    int32_t code, kcode;
    at::ScalarType dt, kdt;
    if (!floats(a[0], 4, d, &code, &dt) || !floats(a[3], 4, c, &kcode, &kdt) || d[1] < 1) Py_RETURN_NONE;
    const int64_t width = size_of(a[5], 2, 1), space = tensor(a[10]) ? tensor(a[10])->numel() : -1;
    spec_rows_t q, k, v, o;
    spec_cache_t cache;
    void *at[6], *workspace, *stream;
    int32_t *table, *ctx, *parent, *count;
    int64_t sq[3], so[3], sk[3], ck[3];
    if (width < 0 || space < 0 || !on.strided(a[0], dt, {d[0], d[1], d[2], d[3]}, sq, &at[0]) ||
        !on.strided(a[1], dt, {d[0], d[1], c[2], d[3]}, sk, &at[1]) || !on.strided(a[2], dt, {d[0], d[1], c[2], d[3]}, sv, &at[2]) ||
        !on.strided(a[3], dt, {c[0], c[1], c[2], d[3]}, ck, &at[3]) || !on.strided(a[4], dt, {c[0], c[1], c[2], d[3]}, cv, &at[4]) ||
        !on.in(a[5], at::kInt, {d[0], width}, &table) || !on.in(a[6], at::kInt, {d[0]}, &ctx) ||
        !on.maybe(a[7], at::kInt, {d[0], d[1] - 1}, &parent) || !on.maybe(a[8], at::kInt, {d[0]}, &count) ||
        !on.strided(a[9], dt, {d[0], d[1], d[2], d[3]}, so, &at[5], true) || !on.in(a[10], at::kByte, {space}, &workspace) ||
        (d[1] > 1 && a[7] == Py_None) || !on.here(a[12]))
      Py_RETURN_NONE;
    for (int i = 0; i < 3; ++i)
      if (sk[i] != sv[i] || ck[i] != cv[i]) Py_RETURN_NONE;
    q = {at[0], sq[0], sq[1], sq[2]}, k = {at[1], sk[0], sk[1], sk[2]}, v = {at[2], sv[0], sv[1], sv[2]}, o = {at[5], so[0], so[1], so[2]};
    cache = {at[3], at[4], ck[0], ck[1], ck[2], (int32_t)c[0], (int32_t)c[1]};
    const float scale = (float)(a[11] == Py_None ? std::pow((double)d[3], -0.5) : PyFloat_AS_DOUBLE(a[11]));
    if (!stream_of(a[12], &stream)) return nullptr;
    return status_of([&] {
      return f_tree_attention(&q, &k, &v, &cache, table, ctx, parent, count, &o, (int32_t)d[0], (int32_t)d[1] - 1, (int32_t)d[2],
                              (int32_t)c[2], (int32_t)d[3], code, (int32_t)width, scale, workspace, space, stream);
    });
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// ctx_len, add, new_len, added, block_table, ring, ring_state, ring_state_new, block_size, row_start, slot, pos, path_row, seq_rows,
// src_row, stream
PyObject* cache_extend(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 16 || (a[12] == Py_None) != (a[14] == Py_None)) Py_RETURN_NONE;
  try {
    const Rows on;
    const int64_t b = size_of(a[4], 2, 0), width = size_of(a[4], 2, 1), blocks = size_of(a[5], 1, 0), cap = size_of(a[10], 1, 0);
    const int64_t path_width = a[12] == Py_None ? 0 : size_of(a[12], 2, 1);
    int32_t *ctx, *add, *len, *added, *table, *ring, *state, *state_new, *start, *slot, *pos, *path, *src, block, seq_rows;
    void* stream;
    if (b < 0 || width < 0 || blocks < 0 || cap < 0 || path_width < 0 || !on.in(a[0], at::kInt, {b}, &ctx) ||
        !on.in(a[1], at::kInt, {b}, &add) || !on.in(a[2], at::kInt, {b}, &len) || !on.in(a[3], at::kInt, {b}, &added) ||
        !on.in(a[4], at::kInt, {b, width}, &table) || !on.in(a[5], at::kInt, {blocks}, &ring) || !on.in(a[6], at::kInt, {2}, &state) ||
        !on.in(a[7], at::kInt, {2}, &state_new) || !int32_of(a[8], &block) || !on.in(a[9], at::kInt, {b + 1}, &start) ||
        !on.in(a[10], at::kInt, {cap}, &slot) || !on.maybe(a[11], at::kInt, {cap}, &pos) ||
        !on.maybe(a[12], at::kInt, {b, path_width}, &path) || !int32_of(a[13], &seq_rows) || !on.maybe(a[14], at::kInt, {cap}, &src) ||
        !on.here(a[15]))
      Py_RETURN_NONE;
    if (!stream_of(a[15], &stream)) return nullptr;
    return status_of([&] {
      return f_cache_extend(ctx, add, len, added, (int32_t)b, table, (int32_t)width, ring, (int32_t)blocks, state, state_new, block, start,
                            slot, pos, src, (int32_t)cap, path, (int32_t)path_width, seq_rows, stream);
    });
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// k_new, v_new, slot, k_cache, v_cache, src_row, stream; layers first in the four, or one layer
PyObject* cache_store(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7) Py_RETURN_NONE;
  try {
    const Rows on;
    int64_t c[5] = {1}, d[4] = {1}, sk[3] = {0}, sv[3] = {0}, ck[4] = {0}, cv[4] = {0};
    int32_t code, kcode;
    at::ScalarType dt, kdt;
    void *at[4], *stream;
    int32_t *slot, *src;
    const int64_t count = size_of(a[2], 1, 0);
    if (floats(a[3], 5, c, &code, &dt)) {
      if (!floats(a[0], 4, d, &kcode, &kdt) || !on.strided(a[0], dt, {c[0], d[1], c[3], c[4]}, sk, &at[0]) ||
          !on.strided(a[1], dt, {c[0], d[1], c[3], c[4]}, sv, &at[1]) || !on.strided(a[3], dt, {c[0], c[1], c[2], c[3], c[4]}, ck, &at[2], true) ||
          !on.strided(a[4], dt, {c[0], c[1], c[2], c[3], c[4]}, cv, &at[3], true))
        Py_RETURN_NONE;
    } else if (floats(a[3], 4, c + 1, &code, &dt)) {
      if (!floats(a[0], 3, d + 1, &kcode, &kdt) || !on.strided(a[0], dt, {d[1], c[3], c[4]}, sk + 1, &at[0]) ||
          !on.strided(a[1], dt, {d[1], c[3], c[4]}, sv + 1, &at[1]) || !on.strided(a[3], dt, {c[1], c[2], c[3], c[4]}, ck + 1, &at[2], true) ||
          !on.strided(a[4], dt, {c[1], c[2], c[3], c[4]}, cv + 1, &at[3], true))
        Py_RETURN_NONE;
    } else {
      Py_RETURN_NONE;
    }
    for (int i = 0; i < 4; ++i)
      if ((i < 3 && sk[i] != sv[i]) || ck[i] != cv[i]) Py_RETURN_NONE;
    if (count < 0 || !on.in(a[2], at::kInt, {count}, &slot) || !on.maybe(a[5], at::kInt, {count}, &src) || !on.here(a[6])) Py_RETURN_NONE;
    const spec_rows_t k = {at[0], sk[0], sk[1], sk[2]}, v = {at[1], sv[0], sv[1], sv[2]};
    const spec_cache_t cache = {at[2], at[3], ck[1], ck[2], ck[3], (int32_t)c[1], (int32_t)c[2]};
    if (!stream_of(a[6], &stream)) return nullptr;
    return status_of([&] {
      return f_cache_store(&k, &v, &cache, ck[0], (int32_t)c[0], (int32_t)d[1], (int32_t)c[3], (int32_t)c[4], code, slot, src,
                           (int32_t)count, stream);
    });
  } catch (...) {
    Py_RETURN_NONE;
  }
}

const char* const kPenalties[] = {"counts", "seen", "repetition", "presence", "frequency", "bias", "bias_row", "allowed", "mask_row"};
PyObject* penalty_names[9];   // interned

bool penalties(const Rows& on, PyObject* dict, int64_t b, int64_t R, int64_t V, spec_penalties_t* pen) {
  if (!PyDict_CheckExact(dict)) return false;
  PyObject *x[9], *key, *value;
  std::fill(std::begin(x), std::end(x), Py_None);
  for (Py_ssize_t at = 0; PyDict_Next(dict, &at, &key, &value);) {
    int i = 0;
    while (i < 9 && key != penalty_names[i]) ++i;
    if (i == 9)   // (a key that was not a literal)
      for (i = 0; i < 9 && !(PyUnicode_CheckExact(key) && PyUnicode_CompareWithASCIIString(key, kPenalties[i]) == 0);) ++i;
    if (i == 9) return false;
    x[i] = value;
  }
  const int64_t W = (V + 31) / 32, n_bias = x[5] == Py_None ? 0 : size_of(x[5], 2, 0), n_allowed = x[7] == Py_None ? 0 : size_of(x[7], 2, 0);
  int32_t *counts, *seen, *bias_row, *allowed, *mask_row;
  float *repetition, *presence, *frequency, *bias;
  if (n_bias < 0 || n_allowed < 0 || (x[5] == Py_None) != (x[6] == Py_None) || (x[7] == Py_None) != (x[8] == Py_None) ||
      !on.maybe(x[0], at::kInt, {b, V}, &counts) || !on.maybe(x[1], at::kInt, {b, W}, &seen) || !on.maybe(x[2], at::kFloat, {b}, &repetition) ||
      !on.maybe(x[3], at::kFloat, {b}, &presence) || !on.maybe(x[4], at::kFloat, {b}, &frequency) ||
      !on.maybe(x[5], at::kFloat, {n_bias, V}, &bias) || !on.maybe(x[6], at::kInt, {b}, &bias_row) ||
      !on.maybe(x[7], at::kInt, {n_allowed, W}, &allowed) || !on.maybe(x[8], at::kInt, {b, R}, &mask_row))
    return false;
  *pen = {counts, reinterpret_cast<uint32_t*>(seen), repetition, presence, frequency, bias, bias_row, reinterpret_cast<uint32_t*>(allowed),
          mask_row, (int32_t)n_bias, (int32_t)n_allowed};
  return true;
}

// logits, out, penalties, node_tok, node_parent, n_nodes, stream
PyObject* penalize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 7 || (a[3] == Py_None) != (a[4] == Py_None)) Py_RETURN_NONE;
  try {
    const Rows on;
    int64_t d[3];
    int32_t code, *tok, *parent, *count;
    at::ScalarType dt;
    void *logits, *out, *stream;
    spec_penalties_t pen;
    if (!floats(a[0], 3, d, &code, &dt) || d[1] < 1 || !on.in(a[0], dt, {d[0], d[1], d[2]}, &logits) ||
        !on.in(a[1], dt, {d[0], d[1], d[2]}, &out) || !penalties(on, a[2], d[0], d[1], d[2], &pen) ||
        !on.maybe(a[3], at::kInt, {d[0], d[1] - 1}, &tok) || !on.maybe(a[4], at::kInt, {d[0], d[1] - 1}, &parent) ||
        !on.maybe(a[5], at::kInt, {d[0]}, &count) || !on.here(a[6]))
      Py_RETURN_NONE;
    if (!stream_of(a[6], &stream)) return nullptr;
    return status_of([&] {
      return f_penalize(logits, code, (int32_t)d[0], (int32_t)d[1] - 1, (int32_t)d[2], &pen, tok, parent, count, out, stream);
    });
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// logits, cand_tokens, cand_node, n_nodes, greedy, accept_len, best_cand, out_tokens, n_out, path_row, accept_all, n_cand, penalties,
// node_tok, node_parent, update, stream
PyObject* verify_tree(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 17 || (a[13] == Py_None) != (a[14] == Py_None) || !PyBool_Check(a[15]) || (a[15] == Py_True && a[12] == Py_None)) Py_RETURN_NONE;
  try {
    const Rows on;
    int64_t d[3];
    int32_t code, *cand, *node, *count, *greedy, *len, *best, *out, *n_out, *path, *all, *n_cand, *tok, *parent;
    at::ScalarType dt;
    void *logits, *stream;
    spec_penalties_t pen = {};
    const int64_t B = size_of(a[1], 3, 1), np = size_of(a[1], 3, 2);
    if (B < 0 || np < 0 || !floats(a[0], 3, d, &code, &dt) || d[1] < 1 || !on.in(a[0], dt, {d[0], d[1], d[2]}, &logits)) Py_RETURN_NONE;
    const int64_t b = d[0], R = d[1];
    if (!on.in(a[1], at::kInt, {b, B, np}, &cand) || !on.in(a[2], at::kInt, {b, B, np}, &node) || !on.maybe(a[3], at::kInt, {b}, &count) ||
        !on.in(a[4], at::kInt, {b, R}, &greedy) || !on.in(a[5], at::kInt, {b}, &len) || !on.in(a[6], at::kInt, {b}, &best) ||
        !on.in(a[7], at::kInt, {b, np + 1}, &out) || !on.in(a[8], at::kInt, {b}, &n_out) || !on.in(a[9], at::kInt, {b, np + 1}, &path) ||
        !on.maybe(a[10], at::kInt, {b, B}, &all) || !on.maybe(a[11], at::kInt, {b}, &n_cand) ||
        (a[12] != Py_None && !penalties(on, a[12], b, R, d[2], &pen)) || !on.maybe(a[13], at::kInt, {b, R - 1}, &tok) ||
        !on.maybe(a[14], at::kInt, {b, R - 1}, &parent) || !on.here(a[16]))
      Py_RETURN_NONE;
    const bool update = a[15] == Py_True;
    if (!stream_of(a[16], &stream)) return nullptr;
    return status_of([&] {
      return f_verify_tree(logits, code, cand, node, n_cand, tok, parent, count, a[12] == Py_None ? nullptr : &pen, (int32_t)b,
                           (int32_t)R - 1, (int32_t)B, (int32_t)np, (int32_t)d[2], greedy, len, best, out, n_out, path, all,
                           update ? const_cast<int32_t*>(pen.counts) : nullptr, update ? const_cast<uint32_t*>(pen.seen) : nullptr, stream);
    });
  } catch (...) {
    Py_RETURN_NONE;
  }
}

// addresses of spec_verify, spec_verify_dynamic, spec_advance, spec_tree_metadata, spec_draft; the binding's stream lookup; addresses
// of spec_tree_attention, spec_cache_extend, spec_cache_store, spec_penalize, spec_verify_tree
PyObject* bind(PyObject*, PyObject* args) {
  unsigned long long v, vd, ad, tm, dr, ta, ce, cs, pe, vt;
  PyObject* s;
  if (!PyArg_ParseTuple(args, "KKKKKOKKKKK", &v, &vd, &ad, &tm, &dr, &s, &ta, &ce, &cs, &pe, &vt)) return nullptr;
  f_verify = reinterpret_cast<decltype(f_verify)>(v);
  f_verify_dynamic = reinterpret_cast<decltype(f_verify_dynamic)>(vd);
  f_advance = reinterpret_cast<decltype(f_advance)>(ad);
  f_tree_metadata = reinterpret_cast<decltype(f_tree_metadata)>(tm);
  f_draft = reinterpret_cast<decltype(f_draft)>(dr);
  f_tree_attention = reinterpret_cast<decltype(f_tree_attention)>(ta);
  f_cache_extend = reinterpret_cast<decltype(f_cache_extend)>(ce);
  f_cache_store = reinterpret_cast<decltype(f_cache_store)>(cs);
  f_penalize = reinterpret_cast<decltype(f_penalize)>(pe);
  f_verify_tree = reinterpret_cast<decltype(f_verify_tree)>(vt);
  for (int i = 0; i < 9; ++i)
    if (!penalty_names[i] && !(penalty_names[i] = PyUnicode_InternFromString(kPenalties[i]))) return nullptr;
  Py_INCREF(s);
  Py_XDECREF(f_stream);
  f_stream = s;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"verify", reinterpret_cast<PyCFunction>(verify), METH_FASTCALL, nullptr},
    {"advance", reinterpret_cast<PyCFunction>(advance), METH_FASTCALL, nullptr},
    {"tree_metadata", reinterpret_cast<PyCFunction>(tree_metadata), METH_FASTCALL, nullptr},
    {"draft", reinterpret_cast<PyCFunction>(draft), METH_FASTCALL, nullptr},
    {"tree_attention", reinterpret_cast<PyCFunction>(tree_attention), METH_FASTCALL, nullptr},
    {"cache_extend", reinterpret_cast<PyCFunction>(cache_extend), METH_FASTCALL, nullptr},
    {"cache_store", reinterpret_cast<PyCFunction>(cache_store), METH_FASTCALL, nullptr},
    {"penalize", reinterpret_cast<PyCFunction>(penalize), METH_FASTCALL, nullptr},
    {"verify_tree", reinterpret_cast<PyCFunction>(verify_tree), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__call() { return PyModule_Create(&module); }
