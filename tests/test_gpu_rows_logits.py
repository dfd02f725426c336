"""spec_penalize and spec_verify_tree against the oracle."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as RO
from paper_2404_19124_amd import binding as B
from tests.rows_common import U16, U32, dev, exact_float, random_parents

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
ALL = ("counts", "seen", "repetition", "presence", "frequency", "bias", "allowed")


def pack(bits):
    """[rows, V] truth values as words of 32, the lowest bit first."""
    rows, V = bits.shape
    full = np.zeros((rows, -(-V // 32) * 32), np.uint64)
    full[:, :V] = bits
    return (full.reshape(rows, -1, 32) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32).view(np.int32)


class Rows:
    """Logits of a batch of trees, whose tokens come back on their own paths, and everything that changes them."""

    def __init__(self, b, M, V, dtype="f32", keep=ALL, seed=0, n_nodes=None, values="random"):
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        self.b, self.M, self.R, self.V, self.dtype = b, M, M + 1, V, DT[dtype]
        x = torch.randn((b, self.R, V), generator=gen) * 3
        if values == "ties":
            x = (x * 2).round()
        self.logits = x.to(self.dtype).cuda()
        self.parent = random_parents(rng, b, M)
        self.tok = rng.integers(0, V, (b, M)).astype(np.int32)
        if M > 1:
            self.tok[:, 1::2] = self.tok[:, :1]     # the same token again and again
        self.n_nodes = np.array(n_nodes if n_nodes is not None else [M - q % 2 * (M > 2) for q in range(b)], np.int32)
        counts = rng.integers(0, 4, (b, V)) * (rng.random((b, V)) < 0.3)
        words = -(-V // 32)
        f = lambda lo, hi: rng.uniform(lo, hi, b).astype(np.float32)
        pen = dict(counts=counts.astype(np.int32), seen=pack((counts > 0) | (rng.random((b, V)) < 0.1)), repetition=f(0.7, 1.5),
                   presence=f(-0.5, 1), frequency=f(-0.3, 0.5))
        pen["bias"], pen["bias_row"] = rng.normal(size=(3, V)).astype(np.float32), rng.integers(-1, 4, b).astype(np.int32)
        pen["allowed"] = rng.integers(0, 1 << 32, (5, words), dtype=np.uint64).astype(np.uint32).view(np.int32)
        pen["mask_row"] = rng.integers(-1, 6, (b, self.R)).astype(np.int32)
        drop = [k for k in ALL if k not in keep] + (["bias_row"] if "bias" not in keep else []) + (["mask_row"] if "allowed" not in keep else [])
        self.pen = {k: v for k, v in pen.items() if k not in drop}

    def dev_pen(self):
        return {k: dev(v) for k, v in self.pen.items()}

    def oracle(self, dt, path=True):
        pen = dict(self.pen)
        for k in ("seen", "allowed"):
            if k in pen:
                pen[k] = pen[k].view(np.uint32)
        with np.errstate(invalid="ignore", over="ignore"):
            return RO.processed(exact_float(self.logits).astype(np.float32), pen, self.tok if path else None, self.parent, self.n_nodes, dt)

    def check_penalized(self, path=True, out=None):
        out = torch.full(self.logits.shape, 7.0, dtype=self.dtype, device="cuda") if out is None else out
        was = out.clone()
        a = (dev(self.tok), dev(self.parent)) if path else (None, None)
        want, sizes = self.oracle(np.float64, path)
        B.spec_penalize(self.logits, out, self.dev_pen(), *a, dev(self.n_nodes))
        torch.cuda.synchronize()
        got, before = exact_float(out), exact_float(was)
        for q in range(self.b):
            n = self.n_nodes[q] + 1
            g, w = got[q, :n], want[q, :n]
            fine = np.isfinite(w)
            assert np.array_equal(fine, np.isfinite(g)) and np.array_equal(g[~fine], w[~fine])
            # every intermediate value is rounded once (a quotient, a product, three differences), the result to its type
            bound = 1.01 * U32 * sizes[q, :n] + (1.01 * U16 * (np.abs(w) + U32 * sizes[q, :n]) if self.dtype == torch.bfloat16 else 0)
            assert (np.abs(g[fine] - w[fine]) <= bound[fine] + 1e-38).all()
            assert np.array_equal(got[q, n:], before[q, n:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,M,V", [(1, 0, 1), (2, 3, 31), (3, 5, 33), (2, 9, 1000), (1, 4, 4099), (5, 0, 2050), (1, 2, 10007)])
def test_penalize(b, M, V, dtype):
    Rows(b, M, V, dtype, seed=V).check_penalized()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,M,V", [(1, 4096, 40), (2, 2500, 9)])
def test_penalize_trees_of_many_nodes(b, M, V, dtype):
    """Up to 4096 nodes, whose parents and tokens lie where the touched chunks are listed afterwards."""
    Rows(b, M, V, dtype, seed=M).check_penalized()


@pytest.mark.parametrize("keep", [(), ("counts",), ("seen",), ("seen", "repetition"), ("counts", "repetition", "presence"), ("bias",), ("allowed",),
                                  ("frequency", "presence", "repetition")])
@pytest.mark.parametrize("path", [False, True])
def test_any_part_may_be_missing(keep, path):
    Rows(2, 6, 300, keep=keep, seed=5).check_penalized(path)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_rows_left_alone(dtype):
    r = Rows(4, 6, 515, dtype, seed=6, n_nodes=[-1, 0, 6, 3])
    keep = r.logits.clone()
    work = r.logits.clone()
    want = torch.full_like(work, 7.0)
    args = (r.dev_pen(), dev(r.tok), dev(r.parent), dev(r.n_nodes))
    B.spec_penalize(keep, want, *args)
    B.spec_penalize(work, work, *args)
    for q, n in enumerate(r.n_nodes):
        assert torch.equal(work[q, :n + 1], want[q, :n + 1]) and torch.equal(work[q, n + 1:], keep[q, n + 1:])
    r.check_penalized()


def test_masked_places_hold_anything_and_infinities_pass():
    r = Rows(2, 3, 200, seed=7, keep=("allowed", "counts", "seen", "repetition"))
    r.pen["mask_row"][:] = 1
    allowed = np.array([[RO.bit(r.pen["allowed"][1].view(np.uint32), t) for t in range(200)]]) > 0
    x = r.logits
    x[:, :, torch.from_numpy(~allowed[0]).cuda()] = float("nan")
    at = np.nonzero(allowed[0])[0]
    x[:, :, at[0]], x[:, :, at[1]] = float("inf"), float("-inf")
    r.check_penalized()


def test_where_seen_is_given_counts_are_looked_at_only_there():
    r = Rows(2, 3, 200, seed=8)
    bits = np.array([[RO.bit(w.view(np.uint32), t) for t in range(200)] for w in r.pen["seen"]]) > 0
    r.pen["counts"][~bits] = 1 << 20
    r.check_penalized()


# ---- verification -----------------------------------------------------------------------------------------------

def tree_of(rng, b, Bc, n, V, M):
    """Candidates with shared prefixes and their nodes in order of first appearance."""
    cand = rng.integers(0, V, (b, Bc, n)).astype(np.int32)
    for p in range(n):
        group = max(1, Bc >> (p + 1))
        cand[:, :, p] = cand[:, (np.arange(Bc) // group) * group, p]
    node, tok, parent = np.zeros_like(cand), np.full((b, M), -1, np.int32), np.full((b, M), -1, np.int32)
    count = []
    for q in range(b):
        seen = {}
        for c in range(Bc):
            for p in range(n):
                key = tuple(cand[q, c, :p + 1])
                if key not in seen:
                    i = seen[key] = len(seen)
                    tok[q, i], parent[q, i] = key[-1], seen.get(key[:-1], -1)
                node[q, c, p] = seen[key]
        count.append(len(seen))
    return cand, node, tok, parent, np.array(count, np.int32)


def run_verify(r, cand, node, n_cand=None, penalties=True, update=False):
    b, Bc, n = cand.shape
    i32 = dict(dtype=torch.int32, device="cuda")
    got = {k: torch.full(s, -9, **i32) for k, s in (("greedy", (b, r.R)), ("accept_len", (b,)), ("best_cand", (b,)),
                                                    ("out_tokens", (b, n + 1)), ("n_out", (b,)), ("path_row", (b, n + 1)),
                                                    ("accept_all", (b, Bc)))}
    pen = r.dev_pen() if penalties else None
    B.spec_verify_tree(r.logits, dev(cand), dev(node), dev(r.n_nodes), got["greedy"], got["accept_len"], got["best_cand"],
                       got["out_tokens"], got["n_out"], got["path_row"], got["accept_all"],
                       None if n_cand is None else dev(np.array(n_cand, np.int32)), pen, dev(r.tok) if penalties else None,
                       dev(r.parent) if penalties else None, update)
    torch.cuda.synchronize()
    return got, pen


def check_verify(r, cand, node, n_cand=None, penalties=True, update=False):
    got, pen = run_verify(r, cand, node, n_cand, penalties, update)
    # (float32, every operation rounded by itself: the same numbers, so the same maximum)
    rows = r.oracle(np.float32)[0] if penalties else exact_float(r.logits)
    want = RO.verify_tree(rows, cand, node, r.n_nodes, n_cand)
    for k, w in want.items():
        assert np.array_equal(got[k].cpu().numpy(), w), k
    if update:
        counts, seen = r.pen["counts"].copy(), r.pen["seen"].copy().view(np.uint32)
        for q in range(r.b):
            for t in want["out_tokens"][q, :want["n_out"][q]]:
                counts[q, t] += 1
                seen[q, t // 32] |= np.uint32(1 << (t % 32))
        assert np.array_equal(pen["counts"].cpu().numpy(), counts) and np.array_equal(pen["seen"].cpu().numpy().view(np.uint32), seen)
    return want


def agreeing(b, Bc, n, V, dtype, seed, M=None, **kw):
    """Rows whose maxima agree with the candidates about two times in three."""
    rng = np.random.default_rng(seed)
    M = Bc * n if M is None else M
    cand, node, tok, parent, count = tree_of(rng, b, Bc, n, V, M)
    r = Rows(b, M, V, dtype, seed=seed, **kw)
    r.tok, r.parent, r.n_nodes = tok, parent, count
    for q in range(b):
        for i in range(count[q]):
            if rng.random() < 0.65:
                row = parent[q, i] + 1
                r.logits[q, row, int(tok[q, i])] = 30.0
                if "mask_row" in r.pen:
                    r.pen["mask_row"][q, row] = -1
    return r, cand, node


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,Bc,n,V", [(1, 1, 1, 7), (3, 4, 3, 100), (2, 16, 3, 1001), (4, 1, 7, 515), (2, 70, 2, 300), (2, 8, 8, 2051)])
@pytest.mark.parametrize("values", ["random", "ties"])
def test_verify(b, Bc, n, V, dtype, values):
    r, cand, node = agreeing(b, Bc, n, V, dtype, seed=b + V, values=values)
    want = check_verify(r, cand, node, update=True)
    if b * n > 2:
        assert want["accept_len"].max() > 0


def test_verify_without_penalties_is_spec_verify_on_shared_rows():
    r, cand, node = agreeing(3, 8, 3, 200, "f32", seed=9, values="ties")
    check_verify(r, cand, node, penalties=False)
    got, _ = run_verify(r, cand, node, penalties=False)
    rows = np.concatenate([np.zeros((3, 8, 1), np.int64), node + 1], 2)
    full = r.logits[torch.arange(3)[:, None, None].cuda(), torch.from_numpy(rows).cuda()].contiguous()
    outs = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((3, 8, 4), (3,), (3,), (3, 4), (3,), (3, 8))]
    B.spec_verify(full, dev(cand), *outs)
    for o, k in zip(outs[1:], ("accept_len", "best_cand", "out_tokens", "n_out", "accept_all")):
        assert torch.equal(o, got[k]), k


def test_candidates_switched_off_idle_sequences_and_padding():
    r, cand, node = agreeing(5, 4, 3, 150, "f32", seed=10)
    r.n_nodes[1], r.n_nodes[2] = -1, 0
    r.logits[1], r.logits[2, 1:] = float("nan"), float("nan")
    cand[3, 2:], node[3, 2:] = -1, -1          # padding as spec_draft_dynamic writes it
    check_verify(r, cand, node, n_cand=[4, 4, 0, 2, 4], update=True)


def test_nodes_out_of_range_are_never_accepted():
    r, cand, node = agreeing(3, 4, 3, 100, "f32", seed=11)
    node[0, 0], node[0, 1, 1], node[1] = 1 << 30, -5, r.n_nodes[1]
    r.n_nodes[2] = 2
    check_verify(r, cand, node)


def test_plain_decoding():
    r = Rows(6, 0, 777, "bf16", seed=12, values="ties")
    none = np.zeros((6, 1, 0), np.int32)
    check_verify(r, none, none, update=True)


def test_rows_with_nothing_to_choose():
    r = Rows(2, 2, 90, seed=13, keep=("allowed", "counts", "seen"))
    r.pen["allowed"][0], r.pen["mask_row"][0] = 0, 0
    r.logits[1, 0], r.logits[1, 1] = float("nan"), float("-inf")
    r.logits[1, 2, 5:] = float("nan")
    r.pen["mask_row"][1] = -1
    cand, node = np.array([[[3, 4]], [[0, 0]]], np.int32), np.array([[[0, 1]], [[0, 1]]], np.int32)
    r.n_nodes[:] = 2
    r.parent[:] = [[-1, 0], [-1, 0]]
    check_verify(r, cand, node)


def test_the_same_token_emitted_twice_counts_twice():
    r = Rows(1, 3, 50, seed=14, keep=("counts", "seen"))
    r.logits[:] = 0
    r.logits[0, :, 7] = 100
    r.tok[:], r.parent[:], r.n_nodes[:] = 7, [[-1, 0, 1]], 3
    cand, node = np.full((1, 1, 3), 7, np.int32), np.array([[[0, 1, 2]]], np.int32)
    before = int(r.pen["counts"][0, 7])
    want = check_verify(r, cand, node, update=True)
    assert want["out_tokens"].tolist() == [[7, 7, 7, 7]]
    got, pen = run_verify(r, cand, node, update=True)
    assert int(pen["counts"][0, 7]) == before + 4


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_large_vocabulary(dtype):
    """Against float32 on the device, one operation after the other (the oracle's loops would take minutes)."""
    r, cand, node = agreeing(2, 4, 3, 128256 + 3, dtype, seed=15, keep=("counts", "seen", "repetition", "bias"))
    got, _ = run_verify(r, cand, node)
    V, pen = r.V, r.dev_pen()
    seen = ((pen["seen"][:, torch.arange(V, device="cuda") // 32] >> (torch.arange(V, device="cuda") % 32)) & 1) > 0
    for q in range(2):
        rows = []
        for row in range(int(r.n_nodes[q]) + 1):
            c = torch.where(seen[q], pen["counts"][q], 0)
            for x in RO.path_of(r.parent[q], row):
                c[int(r.tok[q, x])] += 1
            v, rep = r.logits[q, row].float(), pen["repetition"][q]
            v = torch.where(seen[q] | (c > 0), torch.where(v > 0, v / rep, v * rep), v)
            if 0 <= int(pen["bias_row"][q]) < 3:
                v = v + pen["bias"][int(pen["bias_row"][q])]
            rows.append(int(torch.nonzero(v == v.max())[0]))
        assert got["greedy"][q, :len(rows)].tolist() == rows


# ---- calls of more rows than fit the card at once, whole rows per workgroup, several turns per row --------------------------

def every_row_on_the_device(r):
    """Processed logits in float32 on the device, one operation after the other, without paths."""
    V, pen = r.V, r.dev_pen()
    t = torch.arange(V, device="cuda")
    bit = lambda words: ((words[:, t // 32] >> (t % 32)) & 1) > 0
    seen = bit(pen["seen"])
    c = torch.where(seen, pen["counts"], 0)
    v = r.logits.float()
    per = lambda k: pen[k][:, None, None]
    v = torch.where((seen | (c > 0))[:, None], torch.where(v > 0, v / per("repetition"), v * per("repetition")), v)
    v = v - (pen["frequency"][:, None] * c)[:, None]
    v = torch.where((c > 0)[:, None], v - per("presence"), v)
    row = pen["bias_row"].long()
    v = torch.where(((row >= 0) & (row < 3))[:, None, None], v + pen["bias"][row.clamp(0, 2)][:, None], v)
    row = pen["mask_row"].long()
    ok = bit(pen["allowed"])[row.clamp(0, 4)] | ((row < 0) | (row >= 5))[..., None]
    return torch.where(ok, v, float("-inf"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [8192, 9005])
def test_many_rows(dtype, V):
    r = Rows(40, 29, V, dtype, seed=V, n_nodes=[29 - q % 3 for q in range(40)])
    want = every_row_on_the_device(r)
    out, work = torch.full_like(r.logits, 7.0), r.logits.clone()
    args = (r.dev_pen(), None, None, dev(r.n_nodes))
    B.spec_penalize(r.logits, out, *args)
    B.spec_penalize(work, work, *args)
    B_, n = 2, 3
    cand, node = torch.zeros((40, B_, n), dtype=torch.int32, device="cuda"), torch.zeros((40, B_, n), dtype=torch.int32, device="cuda")
    got = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((40, 30), (40,), (40,), (40, n + 1), (40,), (40, n + 1))]
    B.spec_verify_tree(r.logits, cand, node, dev(r.n_nodes), *got, penalties=args[0])
    for q, m in enumerate(r.n_nodes + 1):
        assert torch.equal(out[q, :m], want[q, :m].to(r.dtype)) and (out[q, m:] == 7).all()
        assert torch.equal(work[q, :m], out[q, :m]) and torch.equal(work[q, m:], r.logits[q, m:])
        best = want[q, :m].max(-1, keepdim=True).values
        first = (want[q, :m] == best).int().argmax(-1)
        assert torch.equal(got[0][q, :m], first.int()) and (got[0][q, m:] == -1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("b,M", [(512, 0), (513, 0), (128, 3), (19, 26), (1, 511), (1, 512)])
def test_where_rows_get_fewer_threads(b, M, dtype):
    """512 rows of a call have 1024 threads each, 513 have 512: the first maxima of both, none on a tie's later place."""
    R, V = M + 1, 8200
    r = Rows(b, M, V, dtype, seed=b, values="ties", n_nodes=[M] * b)
    want = every_row_on_the_device(r)
    got = [torch.full(s, -9, dtype=torch.int32, device="cuda") for s in ((b, R), (b,), (b,), (b, 1), (b,), (b, 1))]
    none = torch.zeros((b, 1, 0), dtype=torch.int32, device="cuda")
    B.spec_verify_tree(r.logits, none, none, dev(r.n_nodes), *got, penalties=r.dev_pen())
    best = want.max(-1, keepdim=True).values
    assert torch.equal(got[0], (want == best).int().argmax(-1).int())
    assert torch.equal(got[3][:, 0], got[0][:, 0]) and (got[1] == 0).all() and (got[4] == 1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_replayed_and_on_another_stream(dtype):
    """The captured call reads what its arguments hold at the replay; a call on another stream while it runs does not disturb it."""
    r, cand, node = agreeing(3, 8, 3, 4099, dtype, seed=31)
    others = [agreeing(3, 8, 3, 4099, dtype, seed=s) for s in (32, 33)]
    a = dict(logits=r.logits.clone(), cand_tokens=dev(cand), cand_node=dev(node), n_nodes=dev(r.n_nodes), node_tok=dev(r.tok),
             node_parent=dev(r.parent), penalties=r.dev_pen())
    new = lambda: {k: torch.full(s, -9, dtype=torch.int32, device="cuda") for k, s in (
        ("greedy", (3, r.R)), ("accept_len", (3,)), ("best_cand", (3,)), ("out_tokens", (3, 4)), ("n_out", (3,)), ("path_row", (3, 4)))}
    got, soft = new(), torch.zeros_like(r.logits)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        B.spec_penalize(a["logits"], soft, a["penalties"], a["node_tok"], a["node_parent"], a["n_nodes"])
        B.spec_verify_tree(**a, **got)
    for x, xc, xn in [(r, cand, node)] + others + [(r, cand, node)]:
        a["logits"].copy_(x.logits)
        for name, t in (("cand_tokens", xc), ("cand_node", xn), ("n_nodes", x.n_nodes), ("node_tok", x.tok), ("node_parent", x.parent)):
            a[name].copy_(dev(t))
        for k, t in x.dev_pen().items():
            a["penalties"][k].copy_(t)
        torch.cuda.synchronize()
        graph.replay()
        mine, eager = new(), torch.full_like(soft, 7.0)
        with torch.cuda.stream(side):
            B.spec_penalize(a["logits"], eager, a["penalties"], a["node_tok"], a["node_parent"], a["n_nodes"])
        B.spec_verify_tree(**a, **mine, stream=side)
        torch.cuda.synchronize()
        assert all(torch.equal(got[k], mine[k]) for k in got)
        want = RO.verify_tree(x.oracle(np.float32)[0], xc, xn, x.n_nodes, None)
        assert all(np.array_equal(got[k].cpu().numpy(), want[k]) for k in got)
        for q, m in enumerate(x.n_nodes + 1):
            assert torch.equal(soft[q, :m], eager[q, :m])
