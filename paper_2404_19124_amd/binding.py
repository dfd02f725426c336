"""ctypes binding of libspecdraft.so: the same names as include/spec.h, argument
marshalling only.  Every step of the path runs in the library's kernels; torch
is used for device memory and the current stream, nothing else.

The library is built in-tree by `python -m paper_2404_19124_amd.build`.  If it
is missing this module raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import torch  # imported before the library is loaded so both share one HIP runtime

SPEC_MAX_STAGES = 8
SPEC_MAX_TOPK = 8
SPEC_MAX_LEAVES = 4096
SPEC_F32, SPEC_BF16 = 0, 1
SPEC_OK, SPEC_EINVAL, SPEC_ESHAPE, SPEC_EDTYPE, SPEC_ENOMEM, SPEC_EHIP = 0, -1, -2, -3, -4, -5

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libspecdraft.so")

EXPORTS = ["spec_create", "spec_destroy", "spec_draft", "spec_draft_static", "spec_draft_dynamic", "spec_verify", "spec_verify_dynamic", "spec_head_logp", "spec_model_scalars",
           "spec_profile_enable", "spec_profile_read", "spec_copy_probe", "spec_tree_metadata", "spec_advance", "spec_tree_attention", "spec_tree_attention_workspace", "spec_cache_extend",
           "spec_cache_store", "spec_penalize", "spec_verify_tree", "spec_plan_contraction", "spec_plan_head", "spec_plan_panel", "spec_last_error", "spec_version"]


class SpecError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("libspecdraft status %d: %s" % (status, message))
        self.status = status


class spec_config_t(C.Structure):
    _fields_ = [("n_predict", C.c_int32), ("emb_dim", C.c_int32), ("inner_dim", C.c_int32), ("vocab", C.c_int32),
                ("weight_dtype", C.c_int32), ("state_weight", C.c_float), ("emb_weight", C.c_float),
                ("ln_eps", C.c_float), ("max_batch", C.c_int32), ("max_top_k", C.c_int32 * SPEC_MAX_STAGES)]


class spec_weights_t(C.Structure):
    _fields_ = [("proj", C.POINTER(C.c_void_p)), ("emb", C.POINTER(C.c_void_p)), ("head", C.POINTER(C.c_void_p)),
                ("ln_gamma", C.POINTER(C.c_void_p)), ("ln_beta", C.POINTER(C.c_void_p))]


class spec_plan_t(C.Structure):
    _fields_ = [(name, C.c_int32) for name in ("kernel", "block_rows", "tile_rows", "row_blocks", "ranges", "tiles",
                                               "parts", "k_split", "workgroups", "lds_bytes", "proj_apart")]


class spec_rows_t(C.Structure):
    _fields_ = [("at", C.c_void_p), ("seq_stride", C.c_int64), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class spec_cache_t(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("block_stride", C.c_int64), ("slot_stride", C.c_int64),
                ("head_stride", C.c_int64), ("n_blocks", C.c_int32), ("block_size", C.c_int32)]


class spec_penalties_t(C.Structure):
    _fields_ = [(name, C.c_void_p) for name in ("counts", "seen", "repetition", "presence", "frequency", "bias", "bias_row",
                                                "allowed", "mask_row")] + [("n_bias", C.c_int32), ("n_allowed", C.c_int32)]


class spec_debug_t(C.Structure):
    _fields_ = [("stage_state", C.c_void_p), ("topk_tok", C.c_void_p), ("topk_logp", C.c_void_p),
                ("row_lse", C.c_void_p)]


class spec_launch_record_t(C.Structure):
    _fields_ = [("kernel", C.c_int32), ("rows", C.c_int32), ("weight_rows", C.c_int32), ("k", C.c_int32),
                ("ms", C.c_float)]


_lib = None


def lib() -> C.CDLL:
    """The loaded library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libspecdraft.so is missing (%s): run `python -m paper_2404_19124_amd.build`; "
                               "there is no fallback path" % LIB_PATH)
        l = C.CDLL(LIB_PATH)
        l.spec_create.restype = C.c_int
        l.spec_create.argtypes = [C.POINTER(spec_config_t), C.POINTER(spec_weights_t), C.c_void_p,
                                  C.POINTER(C.c_void_p)]
        l.spec_destroy.restype = None
        l.spec_destroy.argtypes = [C.c_void_p]
        l.spec_draft.restype = C.c_int
        l.spec_draft.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.c_int32,
                                 C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(spec_debug_t), C.c_void_p]
        l.spec_draft_static.restype = C.c_int
        l.spec_draft_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(C.c_int32), C.c_int32,
                                        C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        l.spec_draft_dynamic.restype = C.c_int
        l.spec_draft_dynamic.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.POINTER(C.c_int32),
                                         C.POINTER(C.c_int32), C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                         C.c_void_p, C.POINTER(spec_debug_t), C.c_void_p]
        l.spec_verify_dynamic.restype = C.c_int
        l.spec_verify_dynamic.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                          C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                          C.c_void_p, C.c_void_p]
        l.spec_verify.restype = C.c_int
        l.spec_verify.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                  C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        l.spec_head_logp.restype = C.c_int
        l.spec_head_logp.argtypes = [C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p]
        l.spec_model_scalars.restype = C.c_int
        l.spec_model_scalars.argtypes = [C.c_void_p, C.POINTER(C.c_float), C.POINTER(C.c_float), C.POINTER(C.c_float)]
        l.spec_profile_enable.restype = C.c_int
        l.spec_profile_enable.argtypes = [C.c_void_p, C.c_int32]
        l.spec_profile_read.restype = C.c_int
        l.spec_profile_read.argtypes = [C.c_void_p, C.POINTER(spec_launch_record_t), C.c_int32, C.POINTER(C.c_int32)]
        l.spec_plan_contraction.restype = C.c_int
        l.spec_plan_contraction.argtypes = [C.c_int32] * 6 + [C.POINTER(spec_plan_t)]
        l.spec_plan_head.restype = C.c_int
        l.spec_plan_head.argtypes = [C.c_int32] * 5 + [C.POINTER(spec_plan_t)]
        l.spec_plan_panel.restype = C.c_int
        l.spec_plan_panel.argtypes = [C.c_int32] * 6 + [C.POINTER(spec_plan_t)]
        l.spec_tree_metadata.restype = C.c_int
        l.spec_tree_metadata.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32] + [C.c_void_p] * 7
        l.spec_advance.restype = C.c_int
        l.spec_advance.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32] + [C.c_void_p] * 6
        rows, cache, pen, i32, ptr = C.POINTER(spec_rows_t), C.POINTER(spec_cache_t), C.POINTER(spec_penalties_t), C.c_int32, C.c_void_p
        l.spec_tree_attention.restype = C.c_int
        l.spec_tree_attention.argtypes = ([rows] * 3 + [cache] + [ptr] * 4 + [rows] + [i32] * 7
                                          + [C.c_float, ptr, C.c_int64, ptr])
        l.spec_tree_attention_workspace.restype = C.c_int
        l.spec_tree_attention_workspace.argtypes = [i32] * 6 + [C.POINTER(C.c_int64)]
        l.spec_cache_extend.restype = C.c_int
        l.spec_cache_extend.argtypes = ([ptr] * 4 + [i32, ptr, i32, ptr, i32, ptr, ptr, i32] + [ptr] * 4
                                        + [i32, ptr, i32, i32, ptr])
        l.spec_cache_store.restype = C.c_int
        l.spec_cache_store.argtypes = [rows, rows, cache, C.c_int64] + [i32] * 5 + [ptr, ptr, i32, ptr]
        l.spec_penalize.restype = C.c_int
        l.spec_penalize.argtypes = [ptr] + [i32] * 4 + [pen] + [ptr] * 5
        l.spec_verify_tree.restype = C.c_int
        l.spec_verify_tree.argtypes = [ptr, i32] + [ptr] * 6 + [pen] + [i32] * 5 + [ptr] * 10
        l.spec_copy_probe.restype = C.c_int
        l.spec_copy_probe.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p]
        l.spec_last_error.restype = C.c_char_p
        l.spec_last_error.argtypes = []
        l.spec_version.restype = C.c_int
        l.spec_version.argtypes = [C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        _lib = l
    return _lib


_fast = None   # the native half of the binding (csrc/call.cpp), once it is loaded


def _native():
    global _fast
    if _fast is None:
        l = lib()
        try:
            from . import _call
        except ImportError as e:
            raise RuntimeError("_call.so is missing or does not load: run `python -m paper_2404_19124_amd.build`; there is no "
                               "fallback path") from e
        at = [C.cast(f, C.c_void_p).value for f in (l.spec_verify, l.spec_verify_dynamic, l.spec_advance, l.spec_tree_metadata,
                                                    l.spec_draft, l.spec_tree_attention, l.spec_cache_extend, l.spec_cache_store,
                                                    l.spec_penalize, l.spec_verify_tree)]
        _call.bind(*at[:5], lambda stream: _stream_ptr(stream), *at[5:])
        _fast = _call
    return _fast


def _done(status: Optional[int]) -> bool:
    """What a native call answered: None = not the usual case, nothing has happened."""
    if status is None:
        return False
    if status:
        _check(status)
    return True


def spec_last_error() -> str:
    return lib().spec_last_error().decode()


def _check(status: int) -> None:
    if status != SPEC_OK:
        raise SpecError(status, spec_last_error())


def spec_version():
    a, b = C.c_int32(), C.c_int32()
    _check(lib().spec_version(C.byref(a), C.byref(b)))
    return a.value, b.value


def _dtype_code(name: str) -> int:
    return {"f32": SPEC_F32, "bf16": SPEC_BF16}[name]


# The current stream's address without a Stream object made only to ask for it, which costs 2 us, a sixth of what a verify takes
# on the host.  Neither is part of torch's public interface, so they may be missing.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream_ptr(stream) -> Optional[int]:
    if stream is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return t.data_ptr() if t is not None else None


_TORCH_DTYPE = {SPEC_F32: torch.float32, SPEC_BF16: torch.bfloat16}
_DTYPE_CODE = {torch.float32: SPEC_F32, torch.bfloat16: SPEC_BF16}
_CHECK_DEVICE = True   # the CPU-only tests of _require switch the device check off to reach the others


def _require(t, name: str, dtype: torch.dtype, shape: Optional[Sequence[int]] = None, optional: bool = False) -> None:
    """Host-side check of a tensor argument before its address crosses the boundary: the library reads
    raw pointers, so a wrong element type, a view with strides or a short buffer would be read (or
    written) out of bounds on the device.  Raises ValueError."""
    # (the usual case in one go: a verify checks a dozen tensors, and its kernels take 9 us)
    if (type(t) is torch.Tensor and t.dtype is dtype and (shape is None or t.shape == shape) and t.is_contiguous()
            and (t.is_cuda or not _CHECK_DEVICE)):
        return
    if t is None:
        if optional:
            return
        raise ValueError("%s is required" % name)
    if not isinstance(t, torch.Tensor):
        raise ValueError("%s must be a torch.Tensor" % name)
    if t.dtype != dtype:
        raise ValueError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    if shape is not None and tuple(t.shape) != tuple(int(x) for x in shape):
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if _CHECK_DEVICE and not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)


def make_config(n_predict, emb_dim, inner_dim, vocab, weight_dtype, max_batch, max_top_k, state_weight=-1.0,
                emb_weight=-1.0, ln_eps=1e-5) -> spec_config_t:
    cfg = spec_config_t()
    cfg.n_predict, cfg.emb_dim, cfg.inner_dim, cfg.vocab = n_predict, emb_dim, inner_dim, vocab
    cfg.weight_dtype = _dtype_code(weight_dtype) if isinstance(weight_dtype, str) else int(weight_dtype)
    cfg.state_weight, cfg.emb_weight, cfg.ln_eps = state_weight, emb_weight, ln_eps
    cfg.max_batch = max_batch
    for i, k in enumerate(list(max_top_k)[:SPEC_MAX_STAGES]):
        cfg.max_top_k[i] = int(k)
    return cfg


class SpecModel:
    """Owner of a spec_model_t*.  Keeps the borrowed tensors alive."""

    def __init__(self, cfg: spec_config_t, weights: Dict[str, List[torch.Tensor]], stream=None):
        n = cfg.n_predict
        self.cfg = cfg
        wdt = _TORCH_DTYPE.get(cfg.weight_dtype)
        if wdt is None:
            raise ValueError("weight_dtype %d is neither SPEC_F32 nor SPEC_BF16" % cfg.weight_dtype)
        for key in ("proj", "emb", "head", "ln_gamma", "ln_beta"):
            if key not in weights or len(weights[key]) != n:
                raise ValueError("weights[%s] needs %d stages" % (key, n))
        for i in range(n):
            in_i = cfg.emb_dim if i == 0 else cfg.inner_dim
            for key, dt, shape in (("proj", wdt, (cfg.inner_dim, in_i)), ("emb", wdt, (cfg.vocab, cfg.inner_dim)),
                                   ("head", wdt, (cfg.vocab, cfg.inner_dim)),
                                   ("ln_gamma", torch.float32, (cfg.inner_dim,)),
                                   ("ln_beta", torch.float32, (cfg.inner_dim,))):
                t = weights[key][i]
                if not isinstance(t, torch.Tensor) or t.dtype != dt or tuple(t.shape) != shape or not t.is_cuda:
                    raise ValueError("weights[%s][%d] must be a device tensor of dtype %s and shape %s"
                                     % (key, i, dt, shape))
        self._keep = {k: [t.contiguous() for t in weights[k]] for k in ("emb", "ln_gamma", "ln_beta")}
        tmp = {k: [t.contiguous() for t in weights[k]] for k in ("proj", "head")}
        w = spec_weights_t()
        arrays = {}
        for key in ("proj", "emb", "head", "ln_gamma", "ln_beta"):
            src = tmp[key] if key in tmp else self._keep[key]
            arr = (C.c_void_p * n)(*[t.data_ptr() for t in src])
            arrays[key] = arr
            setattr(w, key, C.cast(arr, C.POINTER(C.c_void_p)))
        handle = C.c_void_p()
        _check(lib().spec_create(C.byref(cfg), C.byref(w), _stream_ptr(stream), C.byref(handle)))
        self.handle = handle
        del tmp  # proj / head were copied by the library

    def scalars(self):
        a, b, c = C.c_float(), C.c_float(), C.c_float()
        _check(lib().spec_model_scalars(self.handle, C.byref(a), C.byref(b), C.byref(c)))
        return a.value, b.value, c.value

    def close(self):
        if getattr(self, "handle", None):
            lib().spec_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def spec_draft(model: SpecModel, state: torch.Tensor, last_tok: torch.Tensor, top_k: Sequence[int], B: int,
               cand_tokens: torch.Tensor, cand_scores: torch.Tensor, cand_leaf: torch.Tensor,
               dbg: Optional[Dict[str, torch.Tensor]] = None, stream=None) -> None:
    """Enqueues one draft.  All tensors are caller-allocated device tensors."""
    cfg = model.cfg
    if dbg is None and _CHECK_DEVICE and _done((_fast or _native()).draft(
            model.handle.value if model.handle else None, cfg.n_predict, cfg.emb_dim, cfg.weight_dtype, state, last_tok, top_k, B,
            cand_tokens, cand_scores, cand_leaf, stream)):
        return
    n, D = cfg.n_predict, cfg.inner_dim
    wdt = _TORCH_DTYPE[cfg.weight_dtype]
    top_k = [int(k) for k in top_k]
    if len(top_k) != n:
        raise ValueError("top_k needs %d entries, got %d" % (n, len(top_k)))
    if not isinstance(state, torch.Tensor) or state.dim() != 2:
        raise ValueError("state must be a [batch, emb_dim] tensor")
    batch, B = int(state.shape[0]), int(B)
    _require(state, "state", wdt, (batch, cfg.emb_dim))
    _require(last_tok, "last_tok", torch.int32, (batch,))
    _require(cand_tokens, "cand_tokens", torch.int32, (batch, B, n))
    _require(cand_scores, "cand_scores", torch.float32, (batch, B))
    _require(cand_leaf, "cand_leaf", torch.int32, (batch, B))
    if dbg is not None:
        rows, r = [], batch
        for k in top_k:
            rows.append(r)
            r *= max(k, 0)
        sum_rows, sum_rk = sum(rows), sum(r_ * k for r_, k in zip(rows, top_k))
        _require(dbg.get("stage_state"), "dbg[stage_state]", wdt, (sum_rows, D), optional=True)
        _require(dbg.get("topk_tok"), "dbg[topk_tok]", torch.int32, (sum_rk,), optional=True)
        _require(dbg.get("topk_logp"), "dbg[topk_logp]", torch.float32, (sum_rk,), optional=True)
        _require(dbg.get("row_lse"), "dbg[row_lse]", torch.float32, (sum_rows,), optional=True)
    tk = (C.c_int32 * n)(*top_k)
    d = None
    if dbg is not None:
        d = spec_debug_t(_ptr(dbg.get("stage_state")), _ptr(dbg.get("topk_tok")), _ptr(dbg.get("topk_logp")),
                         _ptr(dbg.get("row_lse")))
    _check(lib().spec_draft(model.handle, _ptr(state), _ptr(last_tok), batch, tk, int(B), _ptr(cand_tokens),
                            _ptr(cand_scores), _ptr(cand_leaf), C.byref(d) if d is not None else None,
                            _stream_ptr(stream)))


def spec_draft_static(model: SpecModel, state: torch.Tensor, last_tok: torch.Tensor, top_k: Sequence[int], B: int,
                      cand_tokens: torch.Tensor, cand_scores: torch.Tensor, cand_leaf: torch.Tensor,
                      stream=None) -> None:
    """spec_draft with the call's workspace in the library's static device array (no allocation)."""
    cfg = model.cfg
    n = cfg.n_predict
    wdt = _TORCH_DTYPE[cfg.weight_dtype]
    top_k = [int(k) for k in top_k]
    if len(top_k) != n:
        raise ValueError("top_k needs %d entries, got %d" % (n, len(top_k)))
    if not isinstance(state, torch.Tensor) or state.dim() != 2:
        raise ValueError("state must be a [batch, emb_dim] tensor")
    batch, B = int(state.shape[0]), int(B)
    _require(state, "state", wdt, (batch, cfg.emb_dim))
    _require(last_tok, "last_tok", torch.int32, (batch,))
    _require(cand_tokens, "cand_tokens", torch.int32, (batch, B, n))
    _require(cand_scores, "cand_scores", torch.float32, (batch, B))
    _require(cand_leaf, "cand_leaf", torch.int32, (batch, B))
    tk = (C.c_int32 * n)(*top_k)
    _check(lib().spec_draft_static(model.handle, _ptr(state), _ptr(last_tok), batch, tk, B, _ptr(cand_tokens),
                                   _ptr(cand_scores), _ptr(cand_leaf), _stream_ptr(stream)))


def dynamic_rows(top_k_seq: Sequence[Sequence[int]], B_seq: Sequence[int]):
    """Row bookkeeping of a spec_draft_dynamic call (argument marshalling only): rows per stage over the
    active sequences, the widest branching per stage, and per sequence its first row at every stage."""
    n = len(top_k_seq[0])
    rows, kw, first = [0] * n, [1] * n, []
    for ks, Bq in zip(top_k_seq, B_seq):
        first.append(list(rows))
        if Bq == 0:
            continue
        cnt = 1
        for i, k in enumerate(ks):
            rows[i] += cnt
            kw[i] = max(kw[i], int(k))
            cnt *= int(k)
    return rows, kw, first


def spec_draft_dynamic(model: SpecModel, state: torch.Tensor, last_tok: torch.Tensor,
                       top_k_seq: Sequence[Sequence[int]], B_seq: Sequence[int], cand_tokens: torch.Tensor,
                       cand_scores: torch.Tensor, cand_leaf: torch.Tensor, n_cand: torch.Tensor,
                       dbg: Optional[Dict[str, torch.Tensor]] = None, stream=None) -> None:
    """Enqueues one draft with an own tree (top_k_seq[q]) and candidate count (B_seq[q], 0 = off) per sequence."""
    cfg = model.cfg
    n, D = cfg.n_predict, cfg.inner_dim
    wdt = _TORCH_DTYPE[cfg.weight_dtype]
    if not isinstance(state, torch.Tensor) or state.dim() != 2:
        raise ValueError("state must be a [batch, emb_dim] tensor")
    batch = int(state.shape[0])
    top_k_seq = [[int(k) for k in ks] for ks in top_k_seq]
    B_seq = [int(x) for x in B_seq]
    if len(top_k_seq) != batch or len(B_seq) != batch or any(len(ks) != n for ks in top_k_seq):
        raise ValueError("top_k_seq must be [batch][%d] and B_seq [batch]" % n)
    if not isinstance(cand_tokens, torch.Tensor) or cand_tokens.dim() != 3:
        raise ValueError("cand_tokens must be a [batch, B_pad, n_predict] tensor")
    B_pad = int(cand_tokens.shape[1])
    _require(state, "state", wdt, (batch, cfg.emb_dim))
    _require(last_tok, "last_tok", torch.int32, (batch,))
    _require(cand_tokens, "cand_tokens", torch.int32, (batch, B_pad, n))
    _require(cand_scores, "cand_scores", torch.float32, (batch, B_pad))
    _require(cand_leaf, "cand_leaf", torch.int32, (batch, B_pad))
    _require(n_cand, "n_cand", torch.int32, (batch,))
    d = None
    if dbg is not None:
        rows, kw, _ = dynamic_rows(top_k_seq, B_seq)
        sum_rows, sum_rk = sum(rows), sum(r * k for r, k in zip(rows, kw))
        _require(dbg.get("stage_state"), "dbg[stage_state]", wdt, (sum_rows, D), optional=True)
        _require(dbg.get("topk_tok"), "dbg[topk_tok]", torch.int32, (sum_rk,), optional=True)
        _require(dbg.get("topk_logp"), "dbg[topk_logp]", torch.float32, (sum_rk,), optional=True)
        _require(dbg.get("row_lse"), "dbg[row_lse]", torch.float32, (sum_rows,), optional=True)
        d = spec_debug_t(_ptr(dbg.get("stage_state")), _ptr(dbg.get("topk_tok")), _ptr(dbg.get("topk_logp")),
                         _ptr(dbg.get("row_lse")))
    tk = (C.c_int32 * (batch * n))(*[k for ks in top_k_seq for k in ks])
    bs = (C.c_int32 * batch)(*B_seq)
    _check(lib().spec_draft_dynamic(model.handle, _ptr(state), _ptr(last_tok), batch, tk, bs, B_pad, _ptr(cand_tokens),
                                    _ptr(cand_scores), _ptr(cand_leaf), _ptr(n_cand),
                                    C.byref(d) if d is not None else None, _stream_ptr(stream)))


def spec_verify_dynamic(base_logits: torch.Tensor, cand_tokens: torch.Tensor, n_cand: torch.Tensor,
                        greedy: torch.Tensor, accept_len: torch.Tensor, best_cand: torch.Tensor,
                        out_tokens: torch.Tensor, n_out: torch.Tensor, accept_all: Optional[torch.Tensor] = None,
                        stream=None) -> None:
    """Enqueues one verify in which sequence q has n_cand[q] candidates (0 = speculation off)."""
    if n_cand is not None and _CHECK_DEVICE and _done((_fast or _native()).verify(
            base_logits, cand_tokens, n_cand, greedy, accept_len, best_cand, out_tokens, n_out, accept_all, stream)):
        return
    if not isinstance(base_logits, torch.Tensor) or base_logits.dim() != 4:
        raise ValueError("base_logits must be a [batch, B, n_predict + 1, vocab] tensor")
    b, B, n1, V = base_logits.shape
    code = _DTYPE_CODE.get(base_logits.dtype, -1)
    if code < 0:
        raise ValueError("base_logits must be float32 or bfloat16, got %s" % base_logits.dtype)
    _require(base_logits, "base_logits", base_logits.dtype)
    _require(cand_tokens, "cand_tokens", torch.int32, (b, B, n1 - 1))
    _require(n_cand, "n_cand", torch.int32, (b,))
    _require(greedy, "greedy", torch.int32, (b, B, n1))
    _require(accept_len, "accept_len", torch.int32, (b,))
    _require(best_cand, "best_cand", torch.int32, (b,))
    _require(out_tokens, "out_tokens", torch.int32, (b, n1))
    _require(n_out, "n_out", torch.int32, (b,))
    _require(accept_all, "accept_all", torch.int32, (b, B), optional=True)
    _check(lib().spec_verify_dynamic(_ptr(base_logits), code, _ptr(cand_tokens), _ptr(n_cand), b, B, n1 - 1, V,
                                     _ptr(greedy), _ptr(accept_len), _ptr(best_cand), _ptr(out_tokens), _ptr(n_out),
                                     _ptr(accept_all), _stream_ptr(stream)))


def spec_verify(base_logits: torch.Tensor, cand_tokens: torch.Tensor, greedy: torch.Tensor, accept_len: torch.Tensor,
                best_cand: torch.Tensor, out_tokens: torch.Tensor, n_out: torch.Tensor,
                accept_all: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueues one verify.  base_logits [batch, B, n+1, V] float32 or bfloat16."""
    if _CHECK_DEVICE and _done((_fast or _native()).verify(
            base_logits, cand_tokens, None, greedy, accept_len, best_cand, out_tokens, n_out, accept_all, stream)):
        return
    if not isinstance(base_logits, torch.Tensor) or base_logits.dim() != 4:
        raise ValueError("base_logits must be a [batch, B, n_predict + 1, vocab] tensor")
    b, B, n1, V = base_logits.shape
    code = _DTYPE_CODE.get(base_logits.dtype, -1)
    if code < 0:
        raise ValueError("base_logits must be float32 or bfloat16, got %s" % base_logits.dtype)
    _require(base_logits, "base_logits", base_logits.dtype)
    _require(cand_tokens, "cand_tokens", torch.int32, (b, B, n1 - 1))
    _require(greedy, "greedy", torch.int32, (b, B, n1))
    _require(accept_len, "accept_len", torch.int32, (b,))
    _require(best_cand, "best_cand", torch.int32, (b,))
    _require(out_tokens, "out_tokens", torch.int32, (b, n1))
    _require(n_out, "n_out", torch.int32, (b,))
    _require(accept_all, "accept_all", torch.int32, (b, B), optional=True)
    _check(lib().spec_verify(_ptr(base_logits), code, _ptr(cand_tokens), b, B, n1 - 1, V, _ptr(greedy),
                             _ptr(accept_len), _ptr(best_cand), _ptr(out_tokens), _ptr(n_out), _ptr(accept_all),
                             _stream_ptr(stream)))


def spec_profile_enable(model: SpecModel, capacity: int) -> None:
    _check(lib().spec_profile_enable(model.handle, int(capacity)))


def spec_profile_read(model: SpecModel, cap: int = 65536):
    """Returns a list of dicts (kernel, rows, weight_rows, k, ms), in launch order."""
    buf = (spec_launch_record_t * cap)()
    n = C.c_int32()
    _check(lib().spec_profile_read(model.handle, buf, cap, C.byref(n)))
    return [dict(kernel=r.kernel, rows=r.rows, weight_rows=r.weight_rows, k=r.k, ms=r.ms) for r in buf[:n.value]]


def spec_tree_metadata(cand_tokens: torch.Tensor, node_tok: torch.Tensor, node_parent: torch.Tensor,
                       node_depth: torch.Tensor, n_nodes: torch.Tensor, cand_node: torch.Tensor,
                       mask: Optional[torch.Tensor] = None, stream=None) -> None:
    if _CHECK_DEVICE and _done((_fast or _native()).tree_metadata(cand_tokens, node_tok, node_parent, node_depth, n_nodes, cand_node,
                                                                  mask, stream)):
        return
    if not isinstance(cand_tokens, torch.Tensor) or cand_tokens.dim() != 3:
        raise ValueError("cand_tokens must be a [batch, B, n_predict] tensor")
    b, Bc, n = cand_tokens.shape
    M = Bc * n
    _require(cand_tokens, "cand_tokens", torch.int32)
    _require(node_tok, "node_tok", torch.int32, (b, M))
    _require(node_parent, "node_parent", torch.int32, (b, M))
    _require(node_depth, "node_depth", torch.int32, (b, M))
    _require(n_nodes, "n_nodes", torch.int32, (b,))
    _require(cand_node, "cand_node", torch.int32, (b, Bc, n))
    _require(mask, "mask", torch.uint8, (b, M, M), optional=True)
    _check(lib().spec_tree_metadata(_ptr(cand_tokens), b, Bc, n, _ptr(node_tok), _ptr(node_parent), _ptr(node_depth),
                                    _ptr(n_nodes), _ptr(cand_node), _ptr(mask) if mask is not None else None,
                                    _stream_ptr(stream)))


def spec_advance(hidden: torch.Tensor, best_cand: torch.Tensor, accept_len: torch.Tensor, out_tokens: torch.Tensor,
                 next_state: torch.Tensor, next_tok: torch.Tensor, stream=None) -> None:
    if _CHECK_DEVICE and _done((_fast or _native()).advance(hidden, best_cand, accept_len, out_tokens, next_state, next_tok, stream)):
        return
    if not isinstance(hidden, torch.Tensor) or hidden.dim() != 4:
        raise ValueError("hidden must be a [batch, B, n_predict + 1, emb_dim] tensor")
    b, Bc, n1, E = hidden.shape
    dtype = _DTYPE_CODE.get(hidden.dtype, -1)
    if dtype < 0:
        raise ValueError("hidden must be float32 or bfloat16, got %s" % hidden.dtype)
    _require(hidden, "hidden", hidden.dtype)
    _require(best_cand, "best_cand", torch.int32, (b,))
    _require(accept_len, "accept_len", torch.int32, (b,))
    _require(out_tokens, "out_tokens", torch.int32, (b, n1))
    _require(next_state, "next_state", hidden.dtype, (b, E))
    _require(next_tok, "next_tok", torch.int32, (b,))
    _check(lib().spec_advance(_ptr(hidden), dtype, b, Bc, n1 - 1, E, _ptr(best_cand), _ptr(accept_len),
                              _ptr(out_tokens), _ptr(next_state), _ptr(next_tok), _stream_ptr(stream)))


# ---- around the base model's forward over the token tree: rows of every sequence = the last token, then the tree's nodes ----

def _here(stream, **tensors) -> None:
    """Every tensor that is given lies on the current device, and so does the stream: the kernels run there."""
    if not _CHECK_DEVICE:
        return
    at = None
    for name, t in tensors.items():
        if t is None:
            continue
        if not t.is_cuda:
            raise ValueError("%s must be a device tensor" % name)
        at = torch.cuda.current_device() if at is None else at
        if t.get_device() != at:
            raise ValueError("%s lies on device %d, the current device is %d" % (name, t.get_device(), at))
    on = getattr(stream, "device", None)
    if on is not None and on.index is not None and at is not None and on.index != at:
        raise ValueError("the stream belongs to device %d, the current device is %d" % (on.index, at))


def _float_code(t, name: str, dims: Sequence[int]) -> int:
    if not isinstance(t, torch.Tensor) or t.dim() not in dims:
        raise ValueError("%s must be a tensor of %s dimensions" % (name, " or ".join(str(d) for d in dims)))
    code = _DTYPE_CODE.get(t.dtype, -1)
    if code < 0:
        raise ValueError("%s must be float32 or bfloat16, got %s" % (name, t.dtype))
    return code


def _strided(t, name: str, dtype: torch.dtype, shape: Sequence[int]) -> List[int]:
    """Strides of a tensor whose last dimension is contiguous (0 along dimensions of one entry, whose stride says nothing)."""
    if not isinstance(t, torch.Tensor):
        raise ValueError("%s must be a torch.Tensor" % name)
    if t.dtype != dtype:
        raise ValueError("%s must have dtype %s, got %s" % (name, dtype, t.dtype))
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError("the last dimension of %s must be contiguous" % name)
    return [t.stride(i) if t.shape[i] > 1 else 0 for i in range(t.dim() - 1)]


def _written(t, name: str) -> None:
    """A tensor that is written through strides must not hold an element twice."""
    if any(n > 1 and t.stride(i) == 0 for i, n in enumerate(t.shape)):
        raise ValueError("%s is written and must not be expanded" % name)


def spec_tree_attention_workspace(batch: int, R: int, q_heads: int, kv_heads: int, head_dim: int, dtype: torch.dtype) -> int:
    """Bytes of workspace of spec_tree_attention with R rows per sequence (host-only: needs no GPU)."""
    code = _DTYPE_CODE.get(dtype, -1)
    out = C.c_int64()
    _check(lib().spec_tree_attention_workspace(int(batch), int(R) - 1, int(q_heads), int(kv_heads), int(head_dim), code, C.byref(out)))
    return int(out.value)


def spec_tree_attention(q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, k_cache: torch.Tensor,
                        v_cache: torch.Tensor, block_table: torch.Tensor, ctx_len: torch.Tensor,
                        node_parent: Optional[torch.Tensor], n_nodes: Optional[torch.Tensor], out: torch.Tensor,
                        workspace: torch.Tensor, scale: Optional[float] = None, stream=None) -> None:
    """Enqueues the attention of R = M + 1 rows per sequence over the cache and their own ancestors.

    q, out [batch, R, q_heads, head_dim]; k_new, v_new [batch, R, kv_heads, head_dim]; k_cache, v_cache [n_blocks, block_size,
    kv_heads, head_dim]: any strides but along head_dim, rows on 16 bytes, the same strides in k_* and v_*.  node_parent [batch, M]
    (None: M = 0), n_nodes [batch] (None: M each).  workspace: contiguous uint8, spec_tree_attention_workspace() bytes, not
    shared by calls that may overlap in time.  scale: head_dim ** -0.5 by default.  out may be q."""
    if _CHECK_DEVICE and _done((_fast or _native()).tree_attention(
            q, k_new, v_new, k_cache, v_cache, block_table, ctx_len, node_parent, n_nodes, out, workspace, scale, stream)):
        return
    code = _float_code(q, "q", (4,))
    b, R, H, D = q.shape
    if not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
        raise ValueError("k_cache must be a [n_blocks, block_size, kv_heads, head_dim] tensor")
    if R < 1:
        raise ValueError("q needs a row per sequence")
    if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2:
        raise ValueError("block_table must be a [batch, max_blocks] tensor")
    n_blocks, page, KH, _ = k_cache.shape
    sq, so = _strided(q, "q", q.dtype, (b, R, H, D)), _strided(out, "out", q.dtype, (b, R, H, D))
    sk, sv = _strided(k_new, "k_new", q.dtype, (b, R, KH, D)), _strided(v_new, "v_new", q.dtype, (b, R, KH, D))
    ck = _strided(k_cache, "k_cache", q.dtype, (n_blocks, page, KH, D))
    cv = _strided(v_cache, "v_cache", q.dtype, (n_blocks, page, KH, D))
    if ck != cv or sk != sv:
        raise ValueError("k_cache and v_cache, and k_new and v_new, must have the same strides")
    _written(out, "out")
    M, width = R - 1, int(block_table.shape[1])
    _require(block_table, "block_table", torch.int32, (b, width))
    _require(ctx_len, "ctx_len", torch.int32, (b,))
    _require(node_parent, "node_parent", torch.int32, (b, M), optional=M == 0)
    _require(n_nodes, "n_nodes", torch.int32, (b,), optional=True)
    _require(workspace, "workspace", torch.uint8)
    _here(stream, q=q, out=out, k_new=k_new, v_new=v_new, k_cache=k_cache, v_cache=v_cache, block_table=block_table, ctx_len=ctx_len,
          node_parent=node_parent, n_nodes=n_nodes, workspace=workspace)
    cache = spec_cache_t(_ptr(k_cache), _ptr(v_cache), *ck, n_blocks, page)
    _check(lib().spec_tree_attention(
        C.byref(spec_rows_t(_ptr(q), *sq)), C.byref(spec_rows_t(_ptr(k_new), *sk)), C.byref(spec_rows_t(_ptr(v_new), *sv)),
        C.byref(cache), _ptr(block_table), _ptr(ctx_len), _ptr(node_parent), _ptr(n_nodes), C.byref(spec_rows_t(_ptr(out), *so)),
        b, M, H, KH, D, code, width, D ** -0.5 if scale is None else float(scale), _ptr(workspace) or None, workspace.numel(),
        _stream_ptr(stream)))


def spec_cache_extend(ctx_len: torch.Tensor, add: torch.Tensor, new_len: torch.Tensor, added: torch.Tensor,
                      block_table: torch.Tensor, ring: torch.Tensor, ring_state: torch.Tensor, ring_state_new: torch.Tensor,
                      block_size: int, row_start: torch.Tensor, slot: torch.Tensor, pos: Optional[torch.Tensor] = None,
                      path_row: Optional[torch.Tensor] = None, seq_rows: int = 0, src_row: Optional[torch.Tensor] = None,
                      stream=None) -> None:
    """Enqueues the block tables and slot maps for add[q] tokens more (or fewer) per sequence.

    ctx_len, add, new_len, added [batch]; block_table [batch, max_blocks]; ring [n_blocks]; ring_state, ring_state_new [2];
    row_start [batch + 1]; slot, pos, src_row [cap]; path_row [batch, path_width] with src_row: all int32.  new_len may be
    ctx_len and ring_state_new may be ring_state; no other two may share memory."""
    if _CHECK_DEVICE and _done((_fast or _native()).cache_extend(
            ctx_len, add, new_len, added, block_table, ring, ring_state, ring_state_new, block_size, row_start, slot, pos, path_row, seq_rows,
            src_row, stream)):
        return
    if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2 or not isinstance(ring, torch.Tensor) or ring.dim() != 1:
        raise ValueError("block_table must be a [batch, max_blocks] tensor and ring a [n_blocks] tensor")
    if not isinstance(slot, torch.Tensor) or slot.dim() != 1:
        raise ValueError("slot must be a [cap] tensor")
    (b, width), cap, i32 = block_table.shape, int(slot.shape[0]), torch.int32
    _require(block_table, "block_table", i32)
    for t, name in ((ctx_len, "ctx_len"), (add, "add"), (new_len, "new_len"), (added, "added")):
        _require(t, name, i32, (b,))
    _require(ring, "ring", i32)
    _require(ring_state, "ring_state", i32, (2,))
    _require(ring_state_new, "ring_state_new", i32, (2,))
    _require(row_start, "row_start", i32, (b + 1,))
    _require(slot, "slot", i32)
    _require(pos, "pos", i32, (cap,), optional=True)
    path_width = 0
    if path_row is not None:
        if not isinstance(path_row, torch.Tensor) or path_row.dim() != 2:
            raise ValueError("path_row must be a [batch, path_width] tensor")
        path_width = int(path_row.shape[1])
        _require(path_row, "path_row", i32, (b, path_width))
        _require(src_row, "src_row", i32, (cap,))
    elif src_row is not None:
        raise ValueError("src_row is written with path_row only")
    _here(stream, ctx_len=ctx_len, add=add, new_len=new_len, added=added, block_table=block_table, ring=ring, ring_state=ring_state,
          ring_state_new=ring_state_new, row_start=row_start, slot=slot, pos=pos, path_row=path_row, src_row=src_row)
    _check(lib().spec_cache_extend(_ptr(ctx_len), _ptr(add), _ptr(new_len), _ptr(added), b, _ptr(block_table), width, _ptr(ring),
                                   int(ring.shape[0]), _ptr(ring_state), _ptr(ring_state_new), int(block_size), _ptr(row_start),
                                   _ptr(slot), _ptr(pos), _ptr(src_row), cap, _ptr(path_row), path_width, int(seq_rows),
                                   _stream_ptr(stream)))


def spec_cache_store(k_new: torch.Tensor, v_new: torch.Tensor, slot: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                     src_row: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueues the copy of rows into their cache slots: row src_row[t] (or t) to slot[t], entries without a slot skipped.

    One layer: k_new, v_new [rows, kv_heads, head_dim], k_cache, v_cache [n_blocks, block_size, kv_heads, head_dim].  Several at
    once: a first dimension of layers in all four.  Strides as for spec_tree_attention; slot, src_row [count] int32."""
    if _CHECK_DEVICE and _done((_fast or _native()).cache_store(
            k_new, v_new, slot, k_cache, v_cache, src_row, stream)):
        return
    code = _float_code(k_cache, "k_cache", (4, 5))
    if not isinstance(k_new, torch.Tensor) or not isinstance(v_new, torch.Tensor) or not isinstance(v_cache, torch.Tensor):
        raise ValueError("k_new, v_new and v_cache must be tensors")
    if k_cache.dim() == 4 and k_new.dim() == 3 and v_new.dim() == 3 and v_cache.dim() == 4:
        k_new, v_new, k_cache, v_cache = (t.unsqueeze(0) for t in (k_new, v_new, k_cache, v_cache))
    if k_new.dim() != 4 or k_cache.dim() != 5:
        raise ValueError("k_new must have one dimension less than k_cache")
    L, n_blocks, page, KH, D = k_cache.shape
    rows = int(k_new.shape[1])
    sk, sv = _strided(k_new, "k_new", k_cache.dtype, (L, rows, KH, D)), _strided(v_new, "v_new", k_cache.dtype, (L, rows, KH, D))
    ck = _strided(k_cache, "k_cache", k_cache.dtype, (L, n_blocks, page, KH, D))
    cv = _strided(v_cache, "v_cache", k_cache.dtype, (L, n_blocks, page, KH, D))
    if ck != cv or sk != sv:
        raise ValueError("k_cache and v_cache, and k_new and v_new, must have the same strides")
    _written(k_cache, "k_cache")
    _written(v_cache, "v_cache")
    if not isinstance(slot, torch.Tensor) or slot.dim() != 1:
        raise ValueError("slot must be a [count] tensor")
    count = int(slot.shape[0])
    _require(slot, "slot", torch.int32, (count,))
    _require(src_row, "src_row", torch.int32, (count,), optional=True)
    _here(stream, k_new=k_new, v_new=v_new, k_cache=k_cache, v_cache=v_cache, slot=slot, src_row=src_row)
    _check(lib().spec_cache_store(C.byref(spec_rows_t(_ptr(k_new), *sk)), C.byref(spec_rows_t(_ptr(v_new), *sv)),
                                  C.byref(spec_cache_t(_ptr(k_cache), _ptr(v_cache), *ck[1:], n_blocks, page)), ck[0], L, rows, KH, D,
                                  code, _ptr(slot), _ptr(src_row), count, _stream_ptr(stream)))


_PENALTIES = ("counts", "seen", "repetition", "presence", "frequency", "bias", "bias_row", "allowed", "mask_row")


def _penalties(pen: Dict[str, torch.Tensor], b: int, R: int, V: int, stream) -> spec_penalties_t:
    for key in pen:
        if key not in _PENALTIES:
            raise ValueError("penalties[%s]: not one of %s" % (key, ", ".join(_PENALTIES)))
    t = {k: pen.get(k) for k in _PENALTIES}
    words, i32, f32 = (V + 31) // 32, torch.int32, torch.float32
    n_bias, n_allowed = (int(t[k].shape[0]) if isinstance(t[k], torch.Tensor) and t[k].dim() == 2 else 0 for k in ("bias", "allowed"))
    for name, dt, shape in (("counts", i32, (b, V)), ("seen", i32, (b, words)), ("repetition", f32, (b,)), ("presence", f32, (b,)),
                            ("frequency", f32, (b,)), ("bias", f32, (n_bias, V)), ("bias_row", i32, (b,)),
                            ("allowed", i32, (n_allowed, words)), ("mask_row", i32, (b, R))):
        _require(t[name], "penalties[%s]" % name, dt, shape, optional=True)
    if (t["bias"] is None) != (t["bias_row"] is None) or (t["allowed"] is None) != (t["mask_row"] is None):
        raise ValueError("bias goes with bias_row, and allowed with mask_row")
    _here(stream, **{"penalties[%s]" % k: v for k, v in t.items()})
    return spec_penalties_t(*[_ptr(t[k]) or None for k in _PENALTIES], n_bias, n_allowed)


def spec_penalize(logits: torch.Tensor, out: torch.Tensor, penalties: Dict[str, torch.Tensor],
                  node_tok: Optional[torch.Tensor] = None, node_parent: Optional[torch.Tensor] = None,
                  n_nodes: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueues penalties, biases and masks on logits [batch, R, vocab] into out (which may be logits).

    penalties: any of counts [batch, vocab] int32, seen [batch, W] int32, repetition / presence / frequency [batch] float32,
    bias [n_bias, vocab] float32 with bias_row [batch] int32, allowed [n_allowed, W] int32 with mask_row [batch, R] int32, where
    W = ceil(vocab / 32) words of 32 bits, the lowest first.  node_tok, node_parent [batch, R - 1]: rows count the tokens on their path."""
    if _CHECK_DEVICE and _done((_fast or _native()).penalize(logits, out, penalties, node_tok, node_parent, n_nodes, stream)):
        return
    code = _float_code(logits, "logits", (3,))
    b, R, V = logits.shape
    if R < 1:
        raise ValueError("logits need a row per sequence")
    _require(logits, "logits", logits.dtype)
    _require(out, "out", logits.dtype, (b, R, V))
    _require(node_tok, "node_tok", torch.int32, (b, R - 1), optional=True)
    _require(node_parent, "node_parent", torch.int32, (b, R - 1), optional=True)
    _require(n_nodes, "n_nodes", torch.int32, (b,), optional=True)
    if (node_tok is None) != (node_parent is None):
        raise ValueError("node_tok and node_parent go together")
    pen = _penalties(penalties, b, R, V, stream)
    _here(stream, logits=logits, out=out, node_tok=node_tok, node_parent=node_parent, n_nodes=n_nodes)
    _check(lib().spec_penalize(_ptr(logits), code, b, R - 1, V, C.byref(pen), _ptr(node_tok) or None, _ptr(node_parent) or None,
                               _ptr(n_nodes), _ptr(out), _stream_ptr(stream)))


def spec_verify_tree(logits: torch.Tensor, cand_tokens: torch.Tensor, cand_node: torch.Tensor, n_nodes: Optional[torch.Tensor],
                     greedy: torch.Tensor, accept_len: torch.Tensor, best_cand: torch.Tensor, out_tokens: torch.Tensor,
                     n_out: torch.Tensor, path_row: torch.Tensor, accept_all: Optional[torch.Tensor] = None,
                     n_cand: Optional[torch.Tensor] = None, penalties: Optional[Dict[str, torch.Tensor]] = None,
                     node_tok: Optional[torch.Tensor] = None, node_parent: Optional[torch.Tensor] = None, update: bool = False,
                     stream=None) -> None:
    """Enqueues one verify on logits [batch, R, vocab] of the tree's rows, with penalties as spec_penalize applies them.

    cand_tokens, cand_node [batch, B, n] (n = 0 and B = 1: plain decoding); greedy [batch, R]; accept_len, best_cand, n_out
    [batch]; out_tokens, path_row [batch, n + 1]; accept_all [batch, B].  update: the emitted tokens are added to
    penalties' counts and seen."""
    if _CHECK_DEVICE and _done((_fast or _native()).verify_tree(
            logits, cand_tokens, cand_node, n_nodes, greedy, accept_len, best_cand, out_tokens, n_out, path_row, accept_all, n_cand,
            penalties, node_tok, node_parent, update, stream)):
        return
    code = _float_code(logits, "logits", (3,))
    b, R, V = logits.shape
    if R < 1:
        raise ValueError("logits need a row per sequence")
    if not isinstance(cand_tokens, torch.Tensor) or cand_tokens.dim() != 3:
        raise ValueError("cand_tokens must be a [batch, B, n_predict] tensor")
    i32, (_, Bc, n) = torch.int32, cand_tokens.shape
    _require(logits, "logits", logits.dtype)
    _require(cand_tokens, "cand_tokens", i32, (b, Bc, n))
    _require(cand_node, "cand_node", i32, (b, Bc, n))
    _require(greedy, "greedy", i32, (b, R))
    for t, name in ((accept_len, "accept_len"), (best_cand, "best_cand"), (n_out, "n_out")):
        _require(t, name, i32, (b,))
    _require(out_tokens, "out_tokens", i32, (b, n + 1))
    _require(path_row, "path_row", i32, (b, n + 1))
    _require(accept_all, "accept_all", i32, (b, Bc), optional=True)
    for t, name in ((n_cand, "n_cand"), (n_nodes, "n_nodes")):
        _require(t, name, i32, (b,), optional=True)
    for t, name in ((node_tok, "node_tok"), (node_parent, "node_parent")):
        _require(t, name, i32, (b, R - 1), optional=True)
    if (node_tok is None) != (node_parent is None):
        raise ValueError("node_tok and node_parent go together")
    pen = None if penalties is None else _penalties(penalties, b, R, V, stream)
    if update and pen is None:
        raise ValueError("update needs penalties")
    _here(stream, logits=logits, cand_tokens=cand_tokens, cand_node=cand_node, n_nodes=n_nodes, greedy=greedy, accept_len=accept_len,
          best_cand=best_cand, out_tokens=out_tokens, n_out=n_out, path_row=path_row, accept_all=accept_all, n_cand=n_cand,
          node_tok=node_tok, node_parent=node_parent)
    _check(lib().spec_verify_tree(
        _ptr(logits), code, _ptr(cand_tokens) or None, _ptr(cand_node) or None, _ptr(n_cand), _ptr(node_tok) or None,
        _ptr(node_parent) or None, _ptr(n_nodes), C.byref(pen) if pen is not None else None, b, R - 1, Bc, n, V, _ptr(greedy),
        _ptr(accept_len), _ptr(best_cand), _ptr(out_tokens), _ptr(n_out), _ptr(path_row), _ptr(accept_all),
        pen.counts if update else None, pen.seen if update else None, _stream_ptr(stream)))


def spec_plan_contraction(rows: int, k: int, n_head: int, k_top: int, n_proj: int, n_cu: int = 256) -> dict:
    """The launch plan of one contraction on the streaming and dense kernels (host-only: needs no GPU)."""
    out = spec_plan_t()
    _check(lib().spec_plan_contraction(int(rows), int(k), int(n_head), int(k_top), int(n_proj), int(n_cu), C.byref(out)))
    return {name: int(getattr(out, name)) for name, _ in spec_plan_t._fields_}


def spec_plan_head(rows: int, k: int, n_head: int, k_top: int, n_cu: int = 256) -> dict:
    """The launch plan of a head that is launched alone for its top-k and that spec_plan_panel leaves (host-only: needs no GPU)."""
    out = spec_plan_t()
    _check(lib().spec_plan_head(int(rows), int(k), int(n_head), int(k_top), int(n_cu), C.byref(out)))
    return {name: int(getattr(out, name)) for name, _ in spec_plan_t._fields_}


def spec_plan_panel(rows: int, k: int, n_head: int, k_top: int, n_proj: int, n_cu: int = 256) -> dict:
    """The launch plan of a draft's head and the projection that rides with it, asked before the others (host-only: needs no GPU)."""
    out = spec_plan_t()
    _check(lib().spec_plan_panel(int(rows), int(k), int(n_head), int(k_top), int(n_proj), int(n_cu), C.byref(out)))
    return {name: int(getattr(out, name)) for name, _ in spec_plan_t._fields_}


def spec_copy_probe(src: torch.Tensor, dst: torch.Tensor, stream=None) -> int:
    """One plain copy launch src -> dst (same byte size); returns the bytes copied."""
    _require(src, "src", src.dtype)
    _require(dst, "dst", dst.dtype)
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes:
        raise ValueError("src and dst differ in size")
    _check(lib().spec_copy_probe(_ptr(src), _ptr(dst), nbytes, _stream_ptr(stream)))
    return nbytes


def spec_head_logp(model: SpecModel, stage: int, states: torch.Tensor, logp: torch.Tensor, stream=None) -> None:
    cfg = model.cfg
    if not isinstance(states, torch.Tensor) or states.dim() != 2:
        raise ValueError("states must be a [rows, inner_dim] tensor")
    _require(states, "states", _TORCH_DTYPE[cfg.weight_dtype], (states.shape[0], cfg.inner_dim))
    _require(logp, "logp", torch.float32, (states.shape[0], cfg.vocab))
    _check(lib().spec_head_logp(model.handle, int(stage), _ptr(states), states.shape[0], _ptr(logp),
                                _stream_ptr(stream)))
