"""What the operators on rows of heads and on a cache of four bits refuse, on the host, before any HIP call: no GPU needed."""
import ctypes as C
import types

import pytest
import torch

from paper_2404_19124_amd import binding as B

STREAM = types.SimpleNamespace(cuda_stream=0)
P = 0x10000    # an aligned address that nobody reads: every call here is refused before


def rows(at=P, seq=1 << 12, row=1 << 8, head=64):
    return B.spec_rows_t(at, seq, row, head)


def turn(**kw):
    return B.spec_rotation_t(*dict(dict(cos=P, sin=P, n_pos=9, rot_dim=64, pairs=0), **kw).values())


def cache(**kw):
    a = dict(k=P, v=P, block_stride=1 << 12, slot_stride=1 << 8, head_stride=64, n_blocks=4, block_size=16)
    return B.spec_cache_t(*dict(a, **kw).values())


def packed(**kw):
    a = dict(k=P, v=P, k_scale=P + 1, v_scale=P + 3, block_stride=1 << 10, slot_stride=64, head_stride=32, scale_block_stride=1 << 7, scale_slot_stride=4,
             scale_head_stride=2, n_blocks=4, block_size=16)
    return B.spec_packed_t(*dict(a, **kw).values())


def call(name, a):
    return getattr(B.lib(), name)(*[C.byref(x) if isinstance(x, C.Structure) else x for x in a.values()])


def rotate(**kw):
    a = dict(q=rows(), k=rows(), q_out=rows(), k_out=rows(), batch=2, M=4, q_heads=4, kv_heads=2, head_dim=64, dtype=B.SPEC_BF16, pos=None, ctx_len=P,
             node_depth=P, n_nodes=P, rotation=turn(), q_weight=P, k_weight=P, eps=1e-5, stream=None)
    return call("spec_rotate_rows", dict(a, **kw))


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), B.SPEC_EINVAL), (dict(q_out=rows(at=None)), B.SPEC_EINVAL), (dict(k=None), B.SPEC_EINVAL), (dict(k_out=None), B.SPEC_EINVAL),
    (dict(k=None, k_out=None), B.SPEC_EINVAL),                      # k_weight without k
    (dict(batch=0), B.SPEC_EINVAL), (dict(M=-1), B.SPEC_EINVAL), (dict(q_heads=0), B.SPEC_EINVAL), (dict(kv_heads=0), B.SPEC_EINVAL),
    (dict(q_heads=65536), B.SPEC_ESHAPE), (dict(head_dim=60), B.SPEC_ESHAPE), (dict(head_dim=264), B.SPEC_ESHAPE), (dict(dtype=3), B.SPEC_EDTYPE),
    (dict(batch=1 << 15, M=1 << 11), B.SPEC_ESHAPE), (dict(batch=1, M=0x7fffffff), B.SPEC_ESHAPE), (dict(pos=P), B.SPEC_EINVAL), (dict(ctx_len=None), B.SPEC_EINVAL),
    (dict(node_depth=None), B.SPEC_EINVAL), (dict(rotation=turn(cos=None)), B.SPEC_EINVAL), (dict(rotation=turn(sin=P + 4)), B.SPEC_EINVAL),
    (dict(rotation=turn(n_pos=0)), B.SPEC_EINVAL), (dict(rotation=turn(pairs=2)), B.SPEC_EINVAL), (dict(rotation=turn(rot_dim=0)), B.SPEC_ESHAPE),
    (dict(rotation=turn(rot_dim=72)), B.SPEC_ESHAPE), (dict(rotation=turn(rot_dim=80)), B.SPEC_ESHAPE), (dict(rotation=turn(rot_dim=24)), B.SPEC_ESHAPE),
    (dict(rotation=turn(rot_dim=12), dtype=B.SPEC_F32), B.SPEC_ESHAPE), (dict(q_weight=P + 8), B.SPEC_EINVAL), (dict(eps=-1.0), B.SPEC_EINVAL),
    (dict(eps=float("nan")), B.SPEC_EINVAL), (dict(eps=float("inf")), B.SPEC_EINVAL), (dict(q=rows(row=4)), B.SPEC_EINVAL), (dict(k=rows(at=P + 8)), B.SPEC_EINVAL),
    (dict(q_out=rows(head=32)), B.SPEC_EINVAL), (dict(k_out=rows(row=0)), B.SPEC_EINVAL)])
def test_rotate(kw, status):
    assert rotate(**kw) == status, B.spec_last_error()
    assert B.spec_last_error()


def append(name="spec_cache_append", **kw):
    a = dict(k_new=rows(), v_new=rows(), cache=cache(), layer=1 << 16, layers=2, rows=9, kv_heads=2, head_dim=64, dtype=B.SPEC_BF16, slot=P, src_row=P,
             pos=P, count=5, rotation=turn(), k_weight=P, eps=1e-5, stream=None)
    if name == "spec_packed_append":
        a["cache"] = packed()
        a = {k: v for k, v in a.items() if k != "dtype"}
        at = list(a.items())
        a = dict(at[:4] + [("scale_layer", 1 << 12)] + at[4:])
    return call(name, dict(a, **kw))


BOTH = [
    (dict(k_new=None), B.SPEC_EINVAL), (dict(cache=None), B.SPEC_EINVAL), (dict(v_new=rows(at=None)), B.SPEC_EINVAL), (dict(slot=None), B.SPEC_EINVAL),
    (dict(layers=0), B.SPEC_EINVAL), (dict(layers=65536), B.SPEC_EINVAL), (dict(rows=-1), B.SPEC_EINVAL), (dict(count=-1), B.SPEC_EINVAL),
    (dict(count=(1 << 25) + 1), B.SPEC_ESHAPE), (dict(kv_heads=0), B.SPEC_EINVAL), (dict(kv_heads=65536), B.SPEC_ESHAPE), (dict(head_dim=264), B.SPEC_ESHAPE),
    (dict(pos=None), B.SPEC_EINVAL), (dict(rotation=turn(rot_dim=40)), B.SPEC_ESHAPE), (dict(k_weight=P + 4), B.SPEC_EINVAL), (dict(eps=-0.5), B.SPEC_EINVAL),
    (dict(v_new=rows(seq=1 << 13)), B.SPEC_ESHAPE), (dict(k_new=rows(at=P + 2)), B.SPEC_EINVAL), (dict(layer=4), B.SPEC_EINVAL), (dict(layer=1 << 10), B.SPEC_EINVAL)]


@pytest.mark.parametrize("kw,status", BOTH + [
    (dict(dtype=2), B.SPEC_EDTYPE), (dict(head_dim=20), B.SPEC_ESHAPE), (dict(cache=cache(k=None)), B.SPEC_EINVAL), (dict(cache=cache(n_blocks=0)), B.SPEC_EINVAL),
    (dict(cache=cache(n_blocks=1 << 27)), B.SPEC_ESHAPE), (dict(cache=cache(slot_stride=4)), B.SPEC_EINVAL), (dict(cache=cache(head_stride=32)), B.SPEC_EINVAL)])
def test_append(kw, status):
    assert append(**kw) == status, B.spec_last_error()
    assert B.spec_last_error()


PACKED = [(dict(cache=packed(k_scale=None)), B.SPEC_EINVAL), (dict(cache=packed(v=None)), B.SPEC_EINVAL), (dict(cache=packed(block_size=0)), B.SPEC_EINVAL),
          (dict(cache=packed(n_blocks=1 << 27)), B.SPEC_ESHAPE), (dict(cache=packed(slot_stride=72)), B.SPEC_EINVAL), (dict(cache=packed(v=P + 8)), B.SPEC_EINVAL),
          (dict(head_dim=48), B.SPEC_ESHAPE), (dict(head_dim=0), B.SPEC_ESHAPE)]


@pytest.mark.parametrize("kw,status", BOTH + PACKED + [
    (dict(cache=packed(head_stride=16)), B.SPEC_EINVAL), (dict(cache=packed(scale_head_stride=1)), B.SPEC_EINVAL),
    (dict(cache=packed(scale_slot_stride=0)), B.SPEC_EINVAL), (dict(scale_layer=1 << 8), B.SPEC_EINVAL)])
def test_packed_append(kw, status):
    assert append("spec_packed_append", **kw) == status, B.spec_last_error()
    assert B.spec_last_error()


def load(**kw):
    a = dict(cache=packed(), layer=1 << 16, scale_layer=1 << 12, layers=2, kv_heads=2, head_dim=64, slot=P, count=5, k_out=rows(seq=1 << 14), v_out=rows(seq=1 << 14),
             stream=None)
    return call("spec_packed_load", dict(a, **kw))


@pytest.mark.parametrize("kw,status", PACKED + [
    (dict(k_out=None), B.SPEC_EINVAL), (dict(v_out=rows(at=None, seq=1 << 14)), B.SPEC_EINVAL), (dict(slot=None), B.SPEC_EINVAL), (dict(count=-1), B.SPEC_EINVAL),
    (dict(layers=0), B.SPEC_EINVAL), (dict(kv_heads=0), B.SPEC_EINVAL), (dict(layer=8), B.SPEC_EINVAL), (dict(v_out=rows()), B.SPEC_ESHAPE),
    (dict(k_out=rows(at=P + 8, seq=1 << 14)), B.SPEC_EINVAL), (dict(k_out=rows(seq=1 << 9), v_out=rows(seq=1 << 9)), B.SPEC_EINVAL)])
def test_packed_load(kw, status):
    assert load(**kw) == status, B.spec_last_error()
    assert B.spec_last_error()


def attention(**kw):
    a = dict(q=rows(), k_new=rows(), v_new=rows(), cache=packed(), block_table=P, ctx_len=P, node_parent=P, n_nodes=P, out=rows(), batch=2, M=4, q_heads=4,
             kv_heads=2, head_dim=64, max_blocks=3, scale=1.0, workspace=P, bytes=1 << 40, stream=None)
    return call("spec_packed_attention", dict(a, **kw))


@pytest.mark.parametrize("kw,status", PACKED + [
    (dict(cache=None), B.SPEC_EINVAL), (dict(q=None), B.SPEC_EINVAL), (dict(out=rows(at=None)), B.SPEC_EINVAL), (dict(block_table=None), B.SPEC_EINVAL),
    (dict(ctx_len=None), B.SPEC_EINVAL), (dict(node_parent=None), B.SPEC_EINVAL), (dict(batch=0), B.SPEC_EINVAL), (dict(M=4097), B.SPEC_ESHAPE),
    (dict(q_heads=5), B.SPEC_ESHAPE), (dict(head_dim=288), B.SPEC_ESHAPE), (dict(max_blocks=0), B.SPEC_EINVAL), (dict(max_blocks=1 << 27), B.SPEC_ESHAPE),
    (dict(v_new=rows(seq=1 << 13)), B.SPEC_ESHAPE), (dict(q=rows(at=P + 8)), B.SPEC_EINVAL), (dict(workspace=None), B.SPEC_EINVAL), (dict(bytes=100), B.SPEC_EINVAL),
    (dict(workspace=P + 4), B.SPEC_EINVAL), (dict(out=rows(row=64)), B.SPEC_EINVAL)])
def test_packed_attention(kw, status):
    assert attention(**kw) == status, B.spec_last_error()
    assert B.spec_last_error()


def test_packed_attention_workspace():
    assert B.spec_packed_attention_workspace(2, 5, 4, 2, 64) == B.spec_tree_attention_workspace(2, 5, 4, 2, 64, torch.bfloat16)
    for bad in ((0, 5, 4, 2, 64), (2, 5, 4, 3, 64), (2, 5, 4, 2, 48), (2, 0, 4, 2, 64)):
        with pytest.raises(B.SpecError):
            B.spec_packed_attention_workspace(*bad)
    assert B.lib().spec_packed_attention_workspace(2, 4, 4, 2, 64, None) == B.SPEC_EINVAL


def test_the_binding_checks_tensors(monkeypatch):
    monkeypatch.setattr(B, "_CHECK_DEVICE", False)
    bf, i32, u8 = torch.bfloat16, torch.int32, torch.uint8
    z = lambda *s, t=bf: torch.zeros(s, dtype=t)
    q, k, cos = z(2, 3, 4, 64), z(2, 3, 2, 64), z(9, 32, t=torch.float32)

    def rot(match, **kw):
        a = dict(q=q, k=k, q_out=z(2, 3, 4, 64), k_out=z(2, 3, 2, 64), cos=cos, sin=cos, pos=z(2, 3, t=i32), stream=STREAM)
        with pytest.raises(ValueError, match=match):
            B.spec_rotate_rows(**dict(a, **kw))

    rot("q must be", q=z(3, 4, 64))
    rot("float32 or bfloat16", q=z(2, 3, 4, 64, t=torch.float16))
    rot("k and k_out", k=None)
    rot("k_out must have shape", k_out=z(2, 3, 1, 64))
    rot("q_out must have dtype", q_out=z(2, 3, 4, 64, t=torch.float32))
    rot("must not be expanded", q_out=z(2, 1, 4, 64).expand(2, 3, 4, 64))
    rot("cos and sin", sin=None)
    rot("sin must have shape", sin=cos[:5])
    rot("cos must be contiguous", cos=z(32, 9, t=torch.float32).t())
    rot("pos must have shape", pos=z(2, 4, t=i32))
    rot("node_depth must have shape", node_depth=z(2, 3, t=i32))
    rot("q_weight must have dtype", q_weight=z(64))
    rot("last dimension", q=z(2, 3, 4, 128)[..., ::2])

    new, slot = z(7, 2, 64), z(7, t=i32)

    def app(match, **kw):
        a = dict(k_new=new, v_new=new, slot=slot, k_cache=z(4, 8, 2, 64), v_cache=z(4, 8, 2, 64), pos=slot, cos=cos, sin=cos, stream=STREAM)
        with pytest.raises(ValueError, match=match):
            B.spec_cache_append(**dict(a, **kw))

    app("k_new must have dtype", k_new=new.float())
    app("k_new must be", k_new=z(1, 1, 7, 2, 64))
    app("same strides", v_new=z(7, 3, 64)[:, :2])
    app("same strides", v_cache=z(4, 2, 8, 64).transpose(1, 2))
    app("slot must be", slot=z(7, 1, t=i32))
    app("src_row must have shape", src_row=z(6, t=i32))
    app("pos must have dtype", pos=slot.long())
    app("k_weight must have shape", k_weight=z(32, t=torch.float32))

    def pack(match, load=False, **kw):
        a = dict(k_cache=z(4, 8, 2, 32, t=u8), v_cache=z(4, 8, 2, 32, t=u8), k_scale=z(4, 8, 2, 2, t=u8), v_scale=z(4, 8, 2, 2, t=u8), slot=slot, stream=STREAM)
        a.update(dict(k_out=z(7, 2, 64), v_out=z(7, 2, 64)) if load else dict(k_new=new, v_new=new))
        with pytest.raises(ValueError, match=match):
            (B.spec_packed_load if load else B.spec_packed_append)(**dict(a, **kw))

    for which in (False, True):
        pack("multiple of 32", which, k_cache=z(4, 8, 2, 24, t=u8))
        pack("k_cache must be", which, k_cache=z(8, 2, 32, t=u8))
        pack("v_cache must have dtype", which, v_cache=z(4, 8, 2, 32))
        pack("k_scale must have shape", which, k_scale=z(4, 8, 2, 4, t=u8))
        pack("same strides", which, v_scale=z(4, 8, 4, 2, t=u8)[:, :, :2])
        pack("slot must be", which, slot=None)
    pack("k_new must have dtype", k_new=new.float())
    pack("must not be expanded", k_cache=z(1, 8, 2, 32, t=u8).expand(4, 8, 2, 32), v_cache=z(1, 8, 2, 32, t=u8).expand(4, 8, 2, 32))
    pack("k_out must have shape", True, k_out=z(6, 2, 64))
    pack("same strides", True, v_out=z(2, 7, 64).transpose(0, 1))

    def att(match, **kw):
        a = dict(q=z(2, 3, 4, 64), k_new=z(2, 3, 2, 64), v_new=z(2, 3, 2, 64), k_cache=z(4, 8, 2, 32, t=u8), v_cache=z(4, 8, 2, 32, t=u8), k_scale=z(4, 8, 2, 2, t=u8),
                 v_scale=z(4, 8, 2, 2, t=u8), block_table=z(2, 5, t=i32), ctx_len=z(2, t=i32), node_parent=z(2, 2, t=i32), n_nodes=z(2, t=i32),
                 out=z(2, 3, 4, 64), workspace=z(9, t=u8), stream=STREAM)
        with pytest.raises(ValueError, match=match):
            B.spec_packed_attention(**dict(a, **kw))

    att("q must be a bfloat16", q=z(2, 3, 4, 64, t=torch.float32))
    att("k_cache must be", k_cache=z(1, 4, 8, 2, 32, t=u8))
    att("heads of 64 elements, the cache of 32", **{k: z(4, 8, 2, n, t=u8) for k, n in (("k_cache", 16), ("v_cache", 16), ("k_scale", 1), ("v_scale", 1))})
    att("k_new must have shape", k_new=z(2, 3, 1, 64))
    att("must not be expanded", out=z(2, 1, 4, 64).expand(2, 3, 4, 64))
    att("block_table must be", block_table=z(5, t=i32))
    att("node_parent is required", node_parent=None)
    att("workspace must have dtype", workspace=z(9, t=i32))
