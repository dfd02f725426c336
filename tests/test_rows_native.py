"""The native half of the binding for the operators on a tree's rows: the usual arguments only, the same results as from the
checks one by one, and nothing done where an argument is of another kind."""
from types import SimpleNamespace

import pytest
import torch

from paper_2404_19124_amd import binding as B

NAMES = ("tree_attention", "cache_extend", "cache_store", "penalize", "verify_tree")


def _calls(dev, dtype=torch.float32):
    """(native name, arguments as the native half takes them, entry point, its keyword arguments, what it writes)"""
    g = torch.Generator().manual_seed(11)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    rand = lambda *s: torch.randn(s, generator=g).to(dtype).to(dev)
    b, R, H, KH, D, V = 2, 4, 4, 2, 16, 70
    cache = [rand(6, 8, KH, D) for _ in range(2)]
    new = [rand(b, R, KH, D) for _ in range(2)]
    table, ctx, parent, count = ints([[0, 3], [5, 1]]), ints([11, 3]), ints([[-1, 0, 0], [-1, -1, 1]]), ints([3, 2])
    out = torch.zeros((b, R, H, D), dtype=dtype, device=dev)
    space = torch.empty(B.spec_tree_attention_workspace(b, R, H, KH, D, dtype), dtype=torch.uint8, device=dev)
    att = dict(q=rand(b, R, H, D), k_new=new[0], v_new=new[1], k_cache=cache[0], v_cache=cache[1], block_table=table, ctx_len=ctx,
               node_parent=parent, n_nodes=count, out=out, workspace=space, scale=0.3, stream=None)
    path = ints([[0, 1, 3], [0, 2, -1]])
    ext = dict(ctx_len=ctx, add=ints([3, 2]), new_len=ints([0, 0]), added=ints([0, 0]), block_table=table, ring=ints([2, 4, 0, 0, 0, 0]),
               ring_state=ints([0, 2]), ring_state_new=ints([0, 0]), block_size=8, row_start=ints([0, 0, 0]), slot=ints([-5] * 6),
               pos=ints([-5] * 6), path_row=path, seq_rows=R, src_row=ints([-5] * 6), stream=None)
    layers = [x.unsqueeze(0).repeat(3, *[1] * x.dim()) for x in (new[0].flatten(0, 1), new[1].flatten(0, 1), *cache)]
    store = dict(k_new=layers[0], v_new=layers[1], slot=ints([9, 40, -1, 2]), k_cache=layers[2], v_cache=layers[3], src_row=ints([0, 7, 1, 3]),
                 stream=None)
    one = dict(k_new=new[0].flatten(0, 1), v_new=new[1].flatten(0, 1), slot=ints([9, 40, -1]), k_cache=cache[0].clone(),
               v_cache=cache[1].clone(), src_row=None, stream=None)
    pen = {"counts": torch.randint(0, 2, (b, V), generator=g, dtype=torch.int32).to(dev), "repetition": torch.tensor([1.2, 1.0], device=dev),
           "bias": torch.randn((1, V), generator=g).to(dev), "bias_row": ints([-1, 0]),
           "allowed": torch.full((2, 3), 0x7fff7f7f, dtype=torch.int32, device=dev), "mask_row": ints([[0, -1, 1, 0], [1, 1, -1, 0]])}
    tok = ints([[3, 5, 7], [9, 11, 9]])
    logits = rand(b, R, V)
    pn = dict(logits=logits, out=torch.zeros_like(logits), penalties=pen, node_tok=tok, node_parent=parent, n_nodes=count, stream=None)
    full = lambda *s: torch.full(s, -7, dtype=torch.int32, device=dev)
    ver = dict(logits=logits, cand_tokens=ints([[[3, 5], [3, 7]], [[9, 4], [11, 9]]]), cand_node=ints([[[0, 1], [0, 2]], [[0, 0], [1, 1]]]),
               n_nodes=count, greedy=full(b, R), accept_len=full(b), best_cand=full(b), out_tokens=full(b, 3), n_out=full(b),
               path_row=full(b, 3), accept_all=full(b, 2), n_cand=ints([2, 1]), penalties=dict(pen, counts=pen["counts"].clone()),
               node_tok=tok, node_parent=parent, update=True, stream=None)
    return [
        ("tree_attention", B.spec_tree_attention, att, lambda a: [a["out"][0], a["out"][1, :3]]),
        ("cache_extend", B.spec_cache_extend, ext, lambda a: [a[k] for k in ("new_len", "added", "block_table", "ring", "ring_state_new", "row_start",
                                                                         "slot", "pos", "src_row")]),
        ("cache_store", B.spec_cache_store, store, lambda a: [a["k_cache"], a["v_cache"]]),
        ("cache_store", B.spec_cache_store, one, lambda a: [a["k_cache"], a["v_cache"]]),
        ("penalize", B.spec_penalize, pn, lambda a: [a["out"][0], a["out"][1, :3]]),
        ("verify_tree", B.spec_verify_tree, ver, lambda a: [a[k] for k in ("greedy", "accept_len", "best_cand", "out_tokens", "n_out", "path_row",
                                                                       "accept_all")] + [a["penalties"]["counts"]]),
    ]


def test_nothing_happens_on_host_tensors():
    f = B._native()
    for name, _, args, wrote in _calls("cpu"):
        before = [x.clone() for x in wrote(args)]
        assert getattr(f, name)(*args.values()) is None
        assert getattr(f, name)(*list(args.values())[:-1]) is None        # an argument is missing
        assert getattr(f, name)(*[None] * len(args)) is None
        assert getattr(f, name)(*["x"] * len(args)) is None
        assert all(torch.equal(x, y) for x, y in zip(before, wrote(args)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_both_ways_agree(monkeypatch, dtype):
    fast, slow = _calls("cuda", dtype), _calls("cuda", dtype)
    f = B._native()
    for name, _, args, _ in fast:
        assert getattr(f, name)(*args.values()) == B.SPEC_OK, name
    monkeypatch.setattr(B, "_fast", SimpleNamespace(**{n: lambda *a: None for n in NAMES}))
    for (name, call, args, wrote), (_, _, other, other_wrote) in zip(slow, fast):
        call(**args)
        assert all(torch.equal(x, y) for x, y in zip(wrote(args), other_wrote(other))), name


@pytest.mark.gpu
def test_the_entry_points_take_the_native_way(monkeypatch):
    taken = []
    f = B._native()
    monkeypatch.setattr(B, "_fast", SimpleNamespace(**{n: (lambda n: lambda *a: (taken.append(n), getattr(f, n)(*a))[1])(n) for n in NAMES}))
    for _, call, args, _ in _calls("cuda"):
        call(**args)
    assert taken == ["tree_attention", "cache_extend", "cache_store", "cache_store", "penalize", "verify_tree"]


@pytest.mark.gpu
def test_unusual_arguments_come_back_undone_and_are_refused():
    f = B._native()
    for name, call, args, _ in _calls("cuda"):
        for key, x in args.items():
            if isinstance(x, torch.Tensor):
                for bad in (x.cpu(), x.double() if x.is_floating_point() else x.long(), x[:, None], x.repeat(*[2] * x.dim())):
                    if bad.dtype == x.dtype and bad.is_cuda and (key == "workspace" or key == "ring" and bad.dim() == 1):
                        continue   # (a ring of any length, a workspace of any shape)
                    if key == "slot" and "pos" not in args and args["src_row"] is None and bad.dtype == x.dtype and bad.is_cuda and bad.dim() == 1:
                        continue
                    assert getattr(f, name)(*dict(args, **{key: bad}).values()) is None, (name, key)
                    with pytest.raises(ValueError):
                        call(**dict(args, **{key: bad}))
    att = _calls("cuda")[0][2]
    wide = torch.zeros((2, 4, 2, 32), device="cuda")[..., ::2]
    assert f.tree_attention(*dict(att, k_new=wide).values()) is None
    assert f.tree_attention(*dict(att, out=att["out"][:, :1].expand(2, 4, 4, 16)).values()) is None
    assert f.tree_attention(*dict(att, scale="x").values()) is None
    pen = _calls("cuda")[4][2]
    assert f.penalize(*dict(pen, penalties=dict(pen["penalties"], temperature=1)).values()) is None
    assert f.penalize(*dict(pen, penalties={k: v for k, v in pen["penalties"].items() if k != "bias_row"}).values()) is None
    ver = _calls("cuda")[5][2]
    assert f.verify_tree(*dict(ver, penalties=None).values()) is None      # nothing to update
    assert f.verify_tree(*dict(ver, update=1).values()) is None
