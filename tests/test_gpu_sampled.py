"""spec_verify_sampled against the 64-bit oracle: the same tokens, paths, counts; logarithms of probability in float32."""
import numpy as np
import pytest
import torch

from oracle import sample_oracle as SO
from paper_2404_19124_amd import binding as B
from tests.rows_common import U32, dev, random_parents

pytestmark = pytest.mark.gpu
I32, F32, BF16 = torch.int32, torch.float32, torch.bfloat16


class Case:
    def __init__(self, b, M, V, n, dtype=BF16, seed=0, pen="all", temperature="mixed", n_nodes=None, share=0.6, spread=2.0):
        rng = np.random.default_rng(seed)
        self.b, self.M, self.V, self.n, self.dtype = b, M, V, n, dtype
        R = M + 1
        self.parent = random_parents(rng, b, M, depth=max(n, 1))
        self.tok = np.full((b, M), -1, np.int32)
        for q in range(b):      # siblings differ
            for i in range(M):
                while True:
                    t = int(rng.integers(0, V))
                    if V < 2 * M or not any(self.parent[q, j] == self.parent[q, i] and self.tok[q, j] == t for j in range(i)):
                        break
                self.tok[q, i] = t
        x = spread * rng.normal(size=(b, R, V))
        for q in range(b):      # the drafted tokens have about `share` of their row's mass between them
            for i in range(M):
                x[q, self.parent[q, i] + 1, self.tok[q, i]] = np.log(V) + spread ** 2 / 2 + np.log(share) + rng.normal() * 0.7
        self.logits = torch.from_numpy(x.astype(np.float32)).to(dtype)
        self.n_nodes = None if n_nodes is None else np.array(n_nodes, np.int32)
        self.uniform = rng.random((b, n + 1)).astype(np.float32)
        self.temperature = None if temperature is None else np.where(np.arange(b) % 4 == 3, 0, rng.uniform(0.5, 1.5, b)).astype(np.float32)
        W = -(-V // 32)
        self.pen = None
        if pen:
            said = rng.integers(0, V, (b, max(1, V // 20)))
            counts = np.zeros((b, V), np.int32)
            for q in range(b):
                np.add.at(counts[q], said[q], rng.integers(0, 3, said.shape[1]))
            bits = np.zeros((b, 32 * W), np.uint32)
            for q in range(b):
                bits[q, said[q]] = 1
            full = {"counts": counts, "seen": (bits.reshape(b, W, 32) << np.arange(32, dtype=np.uint32)).sum(2).astype(np.uint32).view(np.int32),
                    "repetition": rng.uniform(1, 1.4, b).astype(np.float32), "presence": rng.uniform(0, 0.5, b).astype(np.float32),
                    "frequency": rng.uniform(0, 0.3, b).astype(np.float32), "bias": (rng.normal(size=(2, V)) * (rng.random((2, V)) < 0.1)).astype(np.float32),
                    "bias_row": rng.integers(-1, 3, b).astype(np.int32),
                    "allowed": rng.integers(-2 ** 31, 2 ** 31, (3, W)).astype(np.int32), "mask_row": rng.integers(-4, 4, (b, R)).astype(np.int32)}
            keys = {"all": list(full), "counts": ["counts", "presence"], "seen": ["seen", "repetition"], "paths": ["frequency", "presence"],
                    "mask": ["allowed", "mask_row"], "bias": ["bias", "bias_row"]}[pen]
            self.pen = {k: full[k] for k in keys}

    def args(self, update=False):
        R = self.M + 1
        space = torch.full((B.spec_verify_sampled_workspace(self.b, R, self.V, self.dtype),), 255, dtype=torch.uint8, device="cuda")
        ints = lambda *s: torch.full(s, -7, dtype=I32, device="cuda")
        return dict(logits=self.logits.cuda(), uniform=dev(self.uniform), n_nodes=None if self.n_nodes is None else dev(self.n_nodes), accept_len=ints(self.b),
                    out_tokens=ints(self.b, self.n + 1), n_out=ints(self.b), path_row=ints(self.b, self.n + 1), workspace=space,
                    out_logp=torch.full((self.b, self.n + 1), 7.0, device="cuda"), temperature=None if self.temperature is None else dev(self.temperature),
                    penalties=None if self.pen is None else {k: dev(v) for k, v in self.pen.items()}, node_tok=dev(self.tok) if self.M else None,
                    node_parent=dev(self.parent) if self.M else None, update=update)

    def check(self, a, update=False, clear=1e-11):
        want = SO.verify(self.logits.float().numpy(), self.tok, self.parent, self.n_nodes, self.temperature, self.uniform, self.pen)
        out, path, logp = a["out_tokens"].cpu().numpy(), a["path_row"].cpu().numpy(), a["out_logp"].cpu().numpy()
        counts = None if self.pen is None or "counts" not in self.pen else self.pen["counts"].copy()
        for q, (tokens, rows, logps, near) in enumerate(want):
            assert near > clear, "the oracle's own sums do not settle sequence %d" % q
            k, pad = len(tokens), [-1] * (self.n + 1 - len(tokens))
            assert out[q].tolist() == tokens + pad, (q, out[q], tokens)
            assert path[q].tolist() == rows + pad, q
            assert int(a["n_out"][q]) == k and int(a["accept_len"][q]) == max(k - 1, 0)
            for i in range(self.n + 1):
                # rounded once; its argument, a quotient of sums, is off by less than 1e-12
                w = logps[i] if i < k else 0.0
                assert logp[q, i] == w or abs(logp[q, i] - w) <= U32 * abs(w) + 1e-11, (q, i)
            if counts is not None:
                np.add.at(counts[q], tokens, 1)
        if update and counts is not None:
            assert np.array_equal(a["penalties"]["counts"].cpu().numpy(), counts)
        if update and self.pen is not None and "seen" in self.pen:
            bits = self.pen["seen"].view(np.uint32).copy()
            for q, (tokens, _, _, _) in enumerate(want):
                for t in tokens:
                    bits[q, t // 32] |= np.uint32(1 << (t % 32))
            assert np.array_equal(a["penalties"]["seen"].cpu().numpy().view(np.uint32), bits)
        return want

    def run(self, update=False):
        a = self.args(update)
        B.spec_verify_sampled(**a)
        torch.cuda.synchronize()
        self.check(a, update)
        return a


CASES = {
    "tree": dict(b=6, M=30, V=3000, n=3), "chain": dict(b=5, M=7, V=32003, n=7), "plain": dict(b=9, M=0, V=5001, n=0), "plain_of_tree": dict(b=4, M=0, V=777, n=4),
    "short_path": dict(b=8, M=40, V=900, n=2, share=0.9), "wide": dict(b=3, M=300, V=4097, n=3, share=0.02), "few_tokens": dict(b=12, M=6, V=9, n=3),
    "seven_tokens": dict(b=12, M=3, V=7, n=3), "one_token": dict(b=3, M=2, V=1, n=2), "idle": dict(b=6, M=12, V=2000, n=4, n_nodes=[-1, 0, 12, 5, -3, 99]),
    "rows_apart": dict(b=3, M=9, V=130000, n=4, share=0.8), "cold": dict(b=6, M=20, V=2500, n=3, spread=12.0), "flat": dict(b=8, M=5, V=9000, n=2, spread=0.0, share=1e-4),
}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("name", CASES)
def test_against_the_oracle(name, dtype):
    for seed in range(3):
        Case(dtype=dtype, seed=seed, **CASES[name]).run(update=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pen", [None, "counts", "seen", "paths", "mask", "bias"])
def test_penalties_one_by_one(pen, dtype):
    Case(7, 25, 1999, 3, dtype, seed=5, pen=pen).run(update=pen in ("counts", "seen"))
    Case(5, 25, 2008, 3, dtype, seed=6, pen=pen, temperature=None).run()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_rows_are_taken_depth_by_depth(dtype):
    """More than 2^24 logits, against the oracle and against the same sequences by themselves: the bits are the same."""
    c = Case(9, 40, 70001, 5, dtype, seed=8, share=0.8, n_nodes=[40, 39, -1, 7, 0, 40, 20, 40, 11])
    a = c.run(update=True)
    assert max(int(x) for x in a["accept_len"]) >= 3
    for q in range(c.b):
        one = c.args()
        for k, x in one.items():
            if isinstance(x, torch.Tensor) and k != "workspace":
                one[k] = x[q:q + 1].contiguous()
        one["penalties"] = {k: x if k in ("bias", "allowed") else x[q:q + 1].contiguous() for k, x in one["penalties"].items()}
        B.spec_verify_sampled(**one)
        for k in ("accept_len", "out_tokens", "n_out", "path_row", "out_logp"):
            assert torch.equal(one[k][0], a[k][q]), (q, k)


def test_vocabularies_of_more_than_64_parts_of_4096():
    Case(2, 3, 300007, 2, BF16, seed=11).run()
    Case(1, 0, 1000003, 0, F32, seed=12).run()


def test_tokens_come_as_often_as_their_probability_says():
    """4096 sequences of the same tree, their random numbers spread evenly: of each token of the first row as many as its share, but for
    one at each end of a stretch."""
    N, V, M = 4096, 50, 4
    c = Case(1, M, V, 1, F32, seed=3, pen=None, temperature=None, spread=1.0)
    c.parent[:] = -1
    c.tok[0] = [7, 0, 49, 23]
    c.b = N
    c.logits, c.tok, c.parent = c.logits.expand(N, -1, -1).contiguous(), np.repeat(c.tok, N, 0), np.repeat(c.parent, N, 0)
    c.uniform = np.stack([(np.arange(N) + 0.5) / N, np.full(N, 0.5)], 1).astype(np.float32)
    a = c.args()
    B.spec_verify_sampled(**a)
    got = np.bincount(a["out_tokens"][:, 0].cpu().numpy(), minlength=V)
    p = SO.weights(c.logits[0, 0].numpy(), 1.0)
    assert (np.abs(got - N * p / p.sum()) <= 2).all()
    went = a["accept_len"].cpu().numpy() == 1
    assert went.sum() == got[[7, 0, 49, 23]].sum() and np.array_equal(a["path_row"][:, 1].cpu().numpy() >= 1, went)


def test_random_numbers_at_and_past_their_ends():
    c = Case(10, 12, 600, 3, F32, seed=4, temperature=None)
    c.uniform[:, :] = np.array([0, 1 - 2.0 ** -24, 1, 1.5, -1, np.nan, np.inf, -np.inf, 2.0 ** -149, 0.5], np.float32)[:, None]
    a = c.args()
    B.spec_verify_sampled(**a)
    c.check(a, clear=-1)   # (0 is the first stretch's beginning)


def test_rows_with_nothing_left_infinite_and_not_a_number():
    c = Case(8, 6, 130, 3, F32, seed=7, pen=None)
    c.parent[:] = np.arange(6) - 1
    c.temperature[:] = [1, 0, 1, 0, 1, 1, 0, 1]
    c.logits[0], c.logits[1] = -np.inf, np.nan
    c.tok[1, :2] = 0                       # a drafted token 0 is the token of a row that has none
    c.logits[2, 0] = -np.inf
    c.logits[2, 0, 77] = -5                # one token left
    c.logits[3, 0, [5, 99]] = np.inf       # the first of two infinite ones
    c.logits[4, 0, [5, 99, 100]] = np.inf  # three that share
    c.tok[4, 0] = 99
    c.logits[5, 0, ::2] = np.nan
    c.logits[6, 0] = np.nan
    c.logits[6, 0, 64] = -np.inf
    c.logits[7, 0] = 3.0e38
    c.logits[7, 0, 3] = -3.0e38
    for u in (0.1, 0.5, 0.9):
        c.uniform[:] = u
        c.run()


def test_siblings_with_the_same_token_and_tokens_that_are_none():
    c = Case(4, 70, 40, 2, BF16, seed=9)       # 70 children of one row among 40 tokens, in two turns of 64
    c.parent[:] = -1
    c.run()
    c.tok[:, ::3], c.tok[:, 1] = -5, 40
    c.tok[:, 4] = 2 ** 31 - 1
    c.run()
    c.parent[:, 5:] = np.arange(5, 70) + 3     # parents that do not come before their nodes: children of row 0
    c.run()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_captured_and_replayed_on_another_stream(dtype):
    for size in (dict(b=5, M=20, V=1500, n=3), dict(b=9, M=40, V=70001, n=4, share=0.8)):
        cases = [Case(dtype=dtype, seed=s, **size) for s in range(3)]
        a = cases[0].args(update=True)
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=side):
            B.spec_verify_sampled(**a)
        for c in cases + cases[:1]:
            fresh = c.args(update=True)
            for k, x in fresh.items():
                if isinstance(x, torch.Tensor):
                    a[k].copy_(x)
            for k, x in fresh["penalties"].items():
                a["penalties"][k].copy_(x)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            c.check(a, update=True)


def test_two_streams_at_once():
    cases = [Case(9, 40, 70001, 4, BF16, seed=s, share=0.8) for s in (20, 21)]
    args = [c.args() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for a, s in zip(args, streams):
            B.spec_verify_sampled(**a, stream=s)
    torch.cuda.synchronize()
    for c, a in zip(cases, args):
        c.check(a)


def test_without_a_temperature_it_is_the_greedy_verification():
    """Tokens and rows as spec_verify_tree's on the tree of the same candidates."""
    rng = np.random.default_rng(31)
    b, Bc, n, V = 5, 6, 3, 400
    cand = dev(rng.integers(0, 5, (b, Bc, n)), I32)
    M = Bc * n
    z = lambda *s: torch.zeros(s, dtype=I32, device="cuda")
    tok, parent, depth, count, node = z(b, M), z(b, M), z(b, M), z(b), z(b, Bc, n)
    B.spec_tree_metadata(cand, tok, parent, depth, count, node, None)
    logits = torch.randn((b, M + 1, V), generator=torch.Generator().manual_seed(2)).cuda()
    logits[:, :, :5] += 4
    greedy = dict(greedy=z(b, M + 1), accept_len=z(b), best_cand=z(b), out_tokens=z(b, n + 1), n_out=z(b), path_row=z(b, n + 1))
    B.spec_verify_tree(logits, cand, node, count, **greedy)
    space = torch.empty(B.spec_verify_sampled_workspace(b, M + 1, V, F32), dtype=torch.uint8, device="cuda")
    got = dict(accept_len=z(b), out_tokens=z(b, n + 1), n_out=z(b), path_row=z(b, n + 1))
    B.spec_verify_sampled(logits, torch.rand((b, n + 1), device="cuda"), count, **got, workspace=space, temperature=torch.zeros(b, device="cuda"), node_tok=tok,
                          node_parent=parent)
    assert int(greedy["accept_len"].max()) > 0
    for k, x in got.items():
        assert torch.equal(x, greedy[k]), k
