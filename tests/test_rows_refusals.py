"""What the operators on a tree's rows refuse, on the host, before any HIP call: no GPU needed."""
import ctypes as C
import types

import pytest
import torch

from paper_2404_19124_amd import binding as B

STREAM = types.SimpleNamespace(cuda_stream=0)
P = 0x10000    # an aligned address that nobody reads: every call here is refused before


def rows(at=P, seq=128, row=64, head=8):
    return B.spec_rows_t(at, seq, row, head)


def cache(**kw):
    a = dict(k=P, v=P, block_stride=256, slot_stride=16, head_stride=8, n_blocks=4, block_size=16)
    a.update(kw)
    return B.spec_cache_t(*a.values())


def attention(**kw):
    a = dict(q=rows(), k_new=rows(), v_new=rows(), cache=cache(), block_table=P, ctx_len=P, node_parent=P, n_nodes=P, out=rows(), batch=2,
             M=4, q_heads=4, kv_heads=2, head_dim=8, dtype=B.SPEC_BF16, max_blocks=3, scale=1.0, workspace=P, bytes=1 << 40, stream=None)
    a.update(kw)
    v = [C.byref(x) if isinstance(x, C.Structure) else x for x in a.values()]
    return B.lib().spec_tree_attention(*v)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), B.SPEC_EINVAL), (dict(out=rows(at=None)), B.SPEC_EINVAL), (dict(cache=cache(v=None)), B.SPEC_EINVAL),
    (dict(block_table=None), B.SPEC_EINVAL), (dict(ctx_len=None), B.SPEC_EINVAL), (dict(node_parent=None), B.SPEC_EINVAL),
    (dict(batch=0), B.SPEC_EINVAL), (dict(M=-1), B.SPEC_EINVAL), (dict(M=4097), B.SPEC_ESHAPE), (dict(q_heads=5), B.SPEC_ESHAPE),
    (dict(kv_heads=0), B.SPEC_EINVAL), (dict(head_dim=12), B.SPEC_ESHAPE), (dict(head_dim=264), B.SPEC_ESHAPE),
    (dict(head_dim=6, dtype=B.SPEC_F32), B.SPEC_ESHAPE), (dict(dtype=2), B.SPEC_EDTYPE), (dict(max_blocks=0), B.SPEC_EINVAL),
    (dict(max_blocks=1 << 27), B.SPEC_ESHAPE), (dict(cache=cache(n_blocks=1 << 27)), B.SPEC_ESHAPE), (dict(cache=cache(block_size=0)), B.SPEC_EINVAL),
    (dict(q=rows(row=4)), B.SPEC_EINVAL), (dict(out=rows(at=P + 8)), B.SPEC_EINVAL), (dict(cache=cache(slot_stride=12)), B.SPEC_EINVAL),
    (dict(v_new=rows(seq=256)), B.SPEC_ESHAPE), (dict(batch=1 << 23, kv_heads=2), B.SPEC_ESHAPE), (dict(workspace=P + 4), B.SPEC_EINVAL),
])
def test_attention(kw, status):
    assert attention(**kw) == status, B.spec_last_error()
    assert B.spec_last_error()


def test_attention_workspace():
    f, out = B.lib().spec_tree_attention_workspace, C.c_int64(-1)
    assert f(1, 4, 4, 2, 8, B.SPEC_BF16, None) == B.SPEC_EINVAL
    assert f(1, 4, 4, 3, 8, B.SPEC_BF16, C.byref(out)) == B.SPEC_ESHAPE and out.value == -1
    for args in ((1, 0, 1, 1, 8, B.SPEC_BF16), (64, 4096, 64, 8, 256, B.SPEC_F32)):
        assert f(*args, C.byref(out)) == B.SPEC_OK
        need = out.value
        assert 0 <= need < 1 << 31
        if need:
            kw = dict(batch=args[0], M=args[1], q_heads=args[2], kv_heads=args[3], head_dim=args[4], dtype=args[5],
                      q=rows(seq=1 << 20, row=1 << 14, head=256), cache=cache(block_stride=1 << 16, slot_stride=1 << 11, head_stride=256))
            assert attention(bytes=need - 1, **kw) == B.SPEC_EINVAL and "workspace" in B.spec_last_error()
            assert attention(workspace=None, **kw) == B.SPEC_EINVAL


def extend(**kw):
    a = dict(ctx_len=P, add=P + 64, new_len=P + 128, added=P + 192, batch=3, block_table=P, max_blocks=4, ring=P, n_blocks=8, ring_state=P,
             ring_state_new=P, block_size=16, row_start=P + 256, slot=P, pos=P, src_row=P, cap=9, path_row=P, path_width=4, seq_rows=5, stream=None)
    a.update(kw)
    return B.lib().spec_cache_extend(*a.values())


@pytest.mark.parametrize("kw,status", [(dict([(k, None)]), B.SPEC_EINVAL) for k in
                                       ("ctx_len", "add", "new_len", "added", "block_table", "ring", "ring_state", "ring_state_new", "row_start", "slot", "src_row")] + [
    (dict(batch=0), B.SPEC_EINVAL), (dict(batch=65536), B.SPEC_EINVAL), (dict(max_blocks=0), B.SPEC_EINVAL), (dict(n_blocks=0), B.SPEC_EINVAL),
    (dict(block_size=0), B.SPEC_EINVAL), (dict(cap=-1), B.SPEC_EINVAL), (dict(cap=(1 << 30) + 1), B.SPEC_ESHAPE),
    (dict(n_blocks=1 << 27), B.SPEC_ESHAPE), (dict(max_blocks=1 << 27), B.SPEC_ESHAPE), (dict(path_width=0), B.SPEC_EINVAL),
    (dict(seq_rows=0), B.SPEC_EINVAL), (dict(batch=60000, seq_rows=60000), B.SPEC_ESHAPE), (dict(added=P), B.SPEC_EINVAL),
    (dict(new_len=P + 64), B.SPEC_EINVAL), (dict(row_start=P), B.SPEC_EINVAL)])
def test_extend(kw, status):
    assert extend(**kw) == status, B.spec_last_error()


def store(**kw):
    a = dict(k_new=rows(), v_new=rows(), cache=cache(), layer=1024, layers=2, n_rows=5, kv_heads=2, head_dim=8, dtype=B.SPEC_BF16, slot=P,
             src_row=P, count=4, stream=None)
    a.update(kw)
    return B.lib().spec_cache_store(*[C.byref(x) if isinstance(x, C.Structure) else x for x in a.values()])


@pytest.mark.parametrize("kw,status", [
    (dict(k_new=None), B.SPEC_EINVAL), (dict(v_new=rows(at=None)), B.SPEC_EINVAL), (dict(slot=None), B.SPEC_EINVAL), (dict(layers=0), B.SPEC_EINVAL),
    (dict(layers=65536), B.SPEC_EINVAL), (dict(n_rows=-1), B.SPEC_EINVAL), (dict(count=-1), B.SPEC_EINVAL), (dict(head_dim=4), B.SPEC_ESHAPE),
    (dict(dtype=7), B.SPEC_EDTYPE), (dict(layer=1020), B.SPEC_EINVAL), (dict(v_new=rows(row=72)), B.SPEC_ESHAPE),
    (dict(cache=cache(head_stride=4)), B.SPEC_EINVAL), (dict(cache=cache(k=None)), B.SPEC_EINVAL), (dict(kv_heads=1 << 24), B.SPEC_ESHAPE)])
def test_store(kw, status):
    assert store(**kw) == status, B.spec_last_error()


def pen(**kw):
    p = B.spec_penalties_t()
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def penalize(**kw):
    a = dict(logits=P, dtype=0, batch=2, M=3, vocab=10, pen=pen(counts=P), node_tok=P, node_parent=P, n_nodes=P, out=P, stream=None)
    a.update(kw)
    return B.lib().spec_penalize(*[C.byref(x) if isinstance(x, C.Structure) else x for x in a.values()])


def verify(**kw):
    a = dict(logits=P, dtype=0, cand=P, node=P, n_cand=None, node_tok=P, node_parent=P, n_nodes=P, pen=None, batch=2, M=3, B=2, n=3, vocab=10,
             greedy=P, accept_len=P, best=P, out=P, n_out=P, path=P, all=None, counts=None, seen=None, stream=None)
    a.update(kw)
    return B.lib().spec_verify_tree(*[C.byref(x) if isinstance(x, C.Structure) else x for x in a.values()])


COMMON = [(dict(logits=None), B.SPEC_EINVAL), (dict(dtype=3), B.SPEC_EDTYPE), (dict(batch=0), B.SPEC_EINVAL), (dict(M=-1), B.SPEC_EINVAL),
          (dict(M=4097), B.SPEC_ESHAPE), (dict(vocab=0), B.SPEC_EINVAL), (dict(vocab=(1 << 30) + 1), B.SPEC_ESHAPE),
          (dict(batch=1 << 30), B.SPEC_ESHAPE), (dict(node_tok=None), B.SPEC_EINVAL), (dict(pen=pen(bias=P)), B.SPEC_EINVAL),
          (dict(pen=pen(allowed=P)), B.SPEC_EINVAL), (dict(pen=pen(bias=P, bias_row=P, n_bias=-1)), B.SPEC_EINVAL)]


@pytest.mark.parametrize("kw,status", COMMON + [(dict(pen=None), B.SPEC_EINVAL), (dict(out=None), B.SPEC_EINVAL)])
def test_penalize(kw, status):
    assert penalize(**kw) == status, B.spec_last_error()


@pytest.mark.parametrize("kw,status", COMMON + [(dict([(k, None)]), B.SPEC_EINVAL) for k in ("cand", "node", "greedy", "accept_len", "best", "out", "n_out", "path")] + [
    (dict(B=0), B.SPEC_EINVAL), (dict(n=-1), B.SPEC_EINVAL), (dict(n=9), B.SPEC_EINVAL), (dict(n=0), B.SPEC_ESHAPE), (dict(B=2000), B.SPEC_ESHAPE)])
def test_verify(kw, status):
    assert verify(**kw) == status, B.spec_last_error()


@pytest.mark.parametrize("call", [penalize, verify])
def test_rows_past_a_launch(call):
    """More rows than workgroups of 512 threads fit a launch of 2^32 threads."""
    for batch, M in (((1 << 23) - 7, 0), (1 << 20, 8), (1 << 15, 256), (2048, 4095)):
        assert call(batch=batch, M=M) == B.SPEC_ESHAPE, (batch, M, B.spec_last_error())


# ---- the binding's own checks -------------------------------------------------------------------------------------

I32 = dict(dtype=torch.int32)


def tensors():
    b, R, H, KH, D, page = 2, 5, 4, 2, 16, 8
    z = lambda *s, **kw: torch.zeros(s, **kw)
    return dict(q=z(b, R, H, D), k_new=z(b, R, KH, D), v_new=z(b, R, KH, D), k_cache=z(6, page, KH, D), v_cache=z(6, page, KH, D),
                block_table=z(b, 3, **I32), ctx_len=z(b, **I32), node_parent=z(b, R - 1, **I32), n_nodes=z(b, **I32), out=z(b, R, H, D),
                workspace=z(1 << 10, dtype=torch.uint8))


@pytest.mark.parametrize("kw,words", [
    (dict(q=torch.zeros((2, 5, 4, 16), dtype=torch.float16)), "float32 or bfloat16"), (dict(q=torch.zeros((2, 5, 64))), "dimensions"),
    (dict(k_new=torch.zeros((2, 5, 3, 16))), "k_new must have shape"), (dict(out=torch.zeros((2, 5, 4, 16), dtype=torch.bfloat16)), "out must have dtype"),
    (dict(v_cache=torch.zeros((6, 2, 8, 16)).transpose(1, 2)), "same strides"), (dict(out=torch.zeros((2, 1, 4, 16)).expand(2, 5, 4, 16)), "expanded"),
    (dict(q=torch.zeros((2, 5, 16, 4)).transpose(2, 3)), "last dimension"), (dict(ctx_len=torch.zeros((2,))), "ctx_len must have dtype"),
    (dict(node_parent=None), "node_parent is required"), (dict(block_table=torch.zeros((3, 3), **I32)), "block_table must have shape"),
    (dict(n_nodes=torch.zeros((3,), **I32)), "n_nodes must have shape"), (dict(workspace=torch.zeros((8,))), "workspace must have dtype"),
    (dict(k_cache=None), "k_cache must be")])
def test_binding_attention(monkeypatch, kw, words):
    with pytest.raises(ValueError, match="device tensor"):
        B.spec_tree_attention(**tensors())
    monkeypatch.setattr(B, "_CHECK_DEVICE", False)
    with pytest.raises(ValueError, match=words):
        B.spec_tree_attention(**dict(tensors(), **kw))


def test_binding_attention_hands_on_what_the_library_refuses(monkeypatch):
    monkeypatch.setattr(B, "_CHECK_DEVICE", False)
    with pytest.raises(B.SpecError):
        B.spec_tree_attention(**dict(tensors(), q=torch.zeros((2, 5, 4, 18))[..., :16], stream=STREAM))    # rows that do not start on 16 bytes
    with pytest.raises(B.SpecError):
        B.spec_tree_attention_workspace(2, 5, 4, 2, 16, torch.float16)


def test_binding_extend(monkeypatch):
    monkeypatch.setattr(B, "_CHECK_DEVICE", False)
    z = lambda *s: torch.zeros(s, **I32)
    a = dict(ctx_len=z(3), add=z(3), new_len=z(3), added=z(3), block_table=z(3, 4), ring=z(8), ring_state=z(2), ring_state_new=z(2), block_size=16,
             row_start=z(4), slot=z(9), pos=z(9), path_row=z(3, 4), seq_rows=5, src_row=z(9))
    for kw, words in ((dict(add=z(4)), "add must have shape"), (dict(row_start=z(3)), "row_start must have shape"), (dict(ring=z(8, 1)), "ring"),
                      (dict(pos=z(8)), "pos must have shape"), (dict(src_row=None), "src_row is required"), (dict(path_row=None), "src_row is written"),
                      (dict(path_row=z(2, 4)), "path_row must have shape"), (dict(slot=torch.zeros((9,))), "slot must have dtype"),
                      (dict(ring_state=z(3)), "ring_state must have shape"), (dict(block_table=z(12)), "block_table must be")):
        with pytest.raises(ValueError, match=words):
            B.spec_cache_extend(**dict(a, **kw))
    with pytest.raises(B.SpecError, match="overlap"):
        B.spec_cache_extend(**dict(a, added=a["ctx_len"], stream=STREAM))


def test_binding_store(monkeypatch):
    monkeypatch.setattr(B, "_CHECK_DEVICE", False)
    z = torch.zeros
    a = dict(k_new=z((2, 5, 2, 16)), v_new=z((2, 5, 2, 16)), slot=z((4,), **I32), k_cache=z((2, 3, 8, 2, 16)), v_cache=z((2, 3, 8, 2, 16)))
    for kw, words in ((dict(k_new=z((5, 2, 16))), "one dimension less"), (dict(v_new=z((2, 5, 3, 16))), "v_new must have shape"),
                      (dict(k_cache=z((2, 3, 8, 2, 16)).half()), "float32 or bfloat16"), (dict(v_cache=z((2, 3, 2, 8, 16)).transpose(2, 3)), "same strides"),
                      (dict(k_cache=z((1, 3, 8, 2, 16)).expand(2, -1, -1, -1, -1), v_cache=z((1, 3, 8, 2, 16)).expand(2, -1, -1, -1, -1)), "expanded"),
                      (dict(src_row=z((5,), **I32)), "src_row must have shape"), (dict(slot=z((4,))), "slot must have dtype")):
        with pytest.raises(ValueError, match=words):
            B.spec_cache_store(**dict(a, **kw))


def test_binding_penalties(monkeypatch):
    monkeypatch.setattr(B, "_CHECK_DEVICE", False)
    z = torch.zeros
    x = z((2, 3, 70))
    for pen_, words in ((dict(count=z((2, 70), **I32)), "not one of"), (dict(counts=z((2, 71), **I32)), "counts"), (dict(seen=z((2, 2), **I32)), "seen"),
                        (dict(bias=z((1, 70))), "bias goes with"), (dict(mask_row=z((2, 3), **I32)), "allowed with"),
                        (dict(repetition=z((2,), dtype=torch.float64)), "repetition"),
                        (dict(allowed=z((4, 3), **I32), mask_row=z((2,), **I32)), "mask_row")):
        with pytest.raises(ValueError, match=words):
            B.spec_penalize(x, x, pen_)
    with pytest.raises(ValueError, match="go together"):
        B.spec_penalize(x, x, {}, node_tok=z((2, 2), **I32))
    with pytest.raises(ValueError, match="out must have dtype"):
        B.spec_penalize(x, x.bfloat16(), {})
    i = lambda *s: z(s, **I32)
    v = dict(logits=x, cand_tokens=i(2, 4, 1), cand_node=i(2, 4, 1), n_nodes=i(2), greedy=i(2, 3), accept_len=i(2), best_cand=i(2), out_tokens=i(2, 2),
             n_out=i(2), path_row=i(2, 2))
    for kw, words in ((dict(cand_node=i(2, 4, 2)), "cand_node"), (dict(greedy=i(2, 2)), "greedy"), (dict(path_row=i(2, 1)), "path_row"),
                      (dict(update=True), "update needs"), (dict(accept_all=i(2, 3)), "accept_all"), (dict(n_cand=i(3)), "n_cand"),
                      (dict(logits=z((2, 3, 70), dtype=torch.half)), "float32 or bfloat16")):
        with pytest.raises(ValueError, match=words):
            B.spec_verify_tree(**dict(v, **kw))


# ---- what is written must not hold an element twice ------------------------------------------------------------------

APART = dict(batch=2, M=4, q_heads=4, kv_heads=2, head_dim=8, workspace=P)


@pytest.mark.parametrize("out", [rows(seq=128, row=64, head=8), rows(seq=512, row=24, head=8), rows(seq=512, row=64, head=0), rows(seq=0, row=64, head=8),
                                 rows(seq=-64, row=64, head=8), rows(seq=32, row=-8, head=80)])
def test_attention_outputs_that_overlap(out):
    """Strides that are not zero and yet lead to the same memory."""
    assert attention(out=out, **APART) == B.SPEC_EINVAL and "overlap" in B.spec_last_error(), B.spec_last_error()


@pytest.mark.parametrize("kw", [dict(layer=0), dict(layer=512), dict(cache=cache(block_stride=128)), dict(cache=cache(slot_stride=8)),
                                dict(cache=cache(slot_stride=-8)), dict(cache=cache(head_stride=0)), dict(cache=cache(block_stride=16, slot_stride=24))])
def test_stores_into_a_cache_that_overlaps(kw):
    assert store(**kw) == B.SPEC_EINVAL and "overlap" in B.spec_last_error(), B.spec_last_error()


def test_binding_refuses_outputs_that_overlap(monkeypatch):
    monkeypatch.setattr(B, "_CHECK_DEVICE", False)
    t = tensors()
    t["workspace"] = torch.zeros(B.spec_tree_attention_workspace(2, 5, 4, 2, 16, torch.float32), dtype=torch.uint8)
    with pytest.raises(B.SpecError, match="rows of out overlap"):
        B.spec_tree_attention(**dict(t, out=torch.zeros(2000).as_strided((2, 5, 4, 16), (320, 32, 16, 1)), stream=STREAM))
    z = torch.zeros
    with pytest.raises(B.SpecError, match="rows of the cache overlap"):
        k = z(2000).as_strided((3, 8, 2, 16), (128, 32, 16, 1))
        B.spec_cache_store(z((5, 2, 16)), z((5, 2, 16)), z((4,), **I32), k, k, stream=STREAM)
