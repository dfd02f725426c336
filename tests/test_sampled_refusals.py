"""What spec_verify_sampled refuses, on the host, before any HIP call, and the native half of its binding (no GPU but where marked)."""
import ctypes as C
import types

import pytest
import torch

from paper_2404_19124_amd import binding as B

P = 0x10000    # an aligned address that nobody reads: every call here is refused before


def verify(**kw):
    a = dict(logits=P, dtype=B.SPEC_BF16, node_tok=P, node_parent=P, n_nodes=P, pen=None, temperature=P, uniform=P, batch=2, M=4, n=3, vocab=100, accept_len=P,
             out_tokens=P, n_out=P, path_row=P, out_logp=P, counts=None, seen=None, workspace=P, bytes=1 << 40, stream=None)
    a.update(kw)
    return B.lib().spec_verify_sampled(*[C.byref(x) if isinstance(x, C.Structure) else x for x in a.values()])


def pen(**kw):
    p = B.spec_penalties_t()
    for k, v in kw.items():
        setattr(p, k, v)
    return p


@pytest.mark.parametrize("kw,status", [(dict([(k, None)]), B.SPEC_EINVAL) for k in
                                       ("logits", "node_tok", "node_parent", "uniform", "accept_len", "out_tokens", "n_out", "path_row", "workspace")] + [
    (dict(node_tok=None, node_parent=None), B.SPEC_EINVAL), (dict(dtype=2), B.SPEC_EDTYPE), (dict(batch=0), B.SPEC_EINVAL), (dict(M=-1), B.SPEC_EINVAL),
    (dict(M=4097), B.SPEC_ESHAPE), (dict(vocab=0), B.SPEC_EINVAL), (dict(vocab=(1 << 30) + 1), B.SPEC_ESHAPE), (dict(n=-1), B.SPEC_EINVAL), (dict(n=9), B.SPEC_EINVAL),
    (dict(batch=(1 << 17) + 1, M=0), B.SPEC_ESHAPE), (dict(batch=1 << 16, M=16), B.SPEC_ESHAPE), (dict(bytes=63), B.SPEC_EINVAL), (dict(workspace=P + 8), B.SPEC_EINVAL),
    (dict(pen=pen(bias=P)), B.SPEC_EINVAL), (dict(pen=pen(allowed=P)), B.SPEC_EINVAL)])
def test_refusals(kw, status):
    assert verify(**kw) == status, B.spec_last_error()
    assert B.spec_last_error()


def test_workspace():
    for b, R, V in ((1, 1, 1), (1, 34, 32000), (32, 65, 128256), (1 << 17, 1, 5), (3, 4097, 300000)):
        for dt in (torch.float32, torch.bfloat16):
            need = B.spec_verify_sampled_workspace(b, R, V, dt)
            assert 0 < need < 1 << 31
            code = B.SPEC_BF16 if dt == torch.bfloat16 else B.SPEC_F32
            assert verify(batch=b, M=R - 1, vocab=V, dtype=code, bytes=need - 1) == B.SPEC_EINVAL and "workspace" in B.spec_last_error()
    for bad in ((0, 1, 1), (1, 0, 1), (1, 4098, 1), (1, 1, 0), ((1 << 17) + 1, 1, 1)):
        with pytest.raises(B.SpecError):
            B.spec_verify_sampled_workspace(*bad, torch.float32)
    with pytest.raises(B.SpecError):
        B.spec_verify_sampled_workspace(1, 1, 1, torch.float16)
    assert B.lib().spec_verify_sampled_workspace(1, 1, 1, 0, None) == B.SPEC_EINVAL


def arguments(dev):
    g = torch.Generator().manual_seed(3)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    b, R, V, n = 2, 4, 70, 2
    full = lambda *s: torch.full(s, -7, dtype=torch.int32, device=dev)
    pens = {"counts": torch.randint(0, 2, (b, V), generator=g, dtype=torch.int32).to(dev), "repetition": torch.tensor([1.2, 1.0], device=dev),
            "allowed": torch.full((2, 3), 0x7fff7f7f, dtype=torch.int32, device=dev), "mask_row": ints([[0, -1, 1, 0], [1, 1, -1, 0]])}
    return dict(logits=torch.randn((b, R, V), generator=g).to(dev), uniform=torch.rand((b, n + 1), generator=g).to(dev), n_nodes=ints([3, 2]), accept_len=full(b),
                out_tokens=full(b, n + 1), n_out=full(b), path_row=full(b, n + 1),
                workspace=torch.empty(B.spec_verify_sampled_workspace(b, R, V, torch.float32), dtype=torch.uint8, device=dev),
                out_logp=torch.full((b, n + 1), 5.0, device=dev), temperature=torch.tensor([0.8, 1.1], device=dev), penalties=pens,
                node_tok=ints([[3, 5, 7], [9, 11, 9]]), node_parent=ints([[-1, 0, 0], [-1, -1, 1]]), update=True, stream=None)


WRITTEN = ("accept_len", "out_tokens", "n_out", "path_row", "out_logp")


def test_the_binding_checks_tensors(monkeypatch):
    f, a = B._native(), arguments("cpu")
    assert f.verify_sampled(*a.values()) is None and f.verify_sampled(*[None] * 15) is None and f.verify_sampled(*["x"] * 15) is None
    assert f.verify_sampled(*list(a.values())[:-1]) is None
    monkeypatch.setattr(B, "_CHECK_DEVICE", False)
    stream = types.SimpleNamespace(cuda_stream=0)

    def bad(match, **kw):
        with pytest.raises(ValueError, match=match):
            B.spec_verify_sampled(**dict(arguments("cpu"), stream=stream, **kw))

    bad("logits must be", logits=torch.zeros((2, 70)))
    bad("uniform must be", uniform=torch.zeros(2))
    bad("uniform must have shape", uniform=torch.zeros((3, 3)))
    bad("uniform must have dtype", uniform=torch.zeros((2, 3), dtype=torch.float64))
    bad("accept_len must have shape", accept_len=torch.zeros(3, dtype=torch.int32))
    bad("path_row must have shape", path_row=torch.zeros((2, 4), dtype=torch.int32))
    bad("out_logp must have dtype", out_logp=torch.zeros((2, 3), dtype=torch.bfloat16))
    bad("temperature must have shape", temperature=torch.zeros(1))
    bad("node_tok is required", node_tok=None)
    bad("node_parent must have dtype", node_parent=torch.zeros((2, 3)))
    bad("workspace is required", workspace=None)
    bad("update needs penalties", penalties=None)
    bad("not one of", penalties={"heat": torch.zeros(2)})


@pytest.mark.gpu
def test_both_ways_agree_and_the_entry_point_takes_the_native_one(monkeypatch):
    f, taken = B._native(), []
    fast, slow, through = (arguments("cuda") for _ in range(3))
    assert f.verify_sampled(*fast.values()) == B.SPEC_OK
    monkeypatch.setattr(B, "_fast", types.SimpleNamespace(verify_sampled=lambda *a: None))
    B.spec_verify_sampled(**slow)
    monkeypatch.setattr(B, "_fast", types.SimpleNamespace(verify_sampled=lambda *a: (taken.append(1), f.verify_sampled(*a))[1]))
    B.spec_verify_sampled(**through)
    assert taken == [1]
    for k in WRITTEN:
        assert torch.equal(fast[k], slow[k]) and torch.equal(fast[k], through[k]), k
    assert torch.equal(fast["penalties"]["counts"], slow["penalties"]["counts"])
    for key, x in fast.items():
        if isinstance(x, torch.Tensor):
            for other in (x.cpu(), x.double(), x[:, None]):
                if key == "workspace" and other.is_cuda and other.dtype == x.dtype:
                    continue
                assert f.verify_sampled(*dict(fast, **{key: other}).values()) is None, key
    assert f.verify_sampled(*dict(fast, update=1).values()) is None and f.verify_sampled(*dict(fast, node_tok=None, node_parent=None).values()) is None
