"""A server's steps over a cache of four bits, eager and captured: prompts are appended, each step turns the rows of a tree, attends, draws
tokens, extends the cache by what was kept and appends it with the rotation on the way; sequences end, and others take their place.  Every
step is checked against the oracles, which get the cache that the sequence's own tokens stand for and not the device's."""
import numpy as np
import pytest
import torch

from oracle import heads_oracle as HO
from oracle import sample_oracle as SO
from paper_2404_19124_amd import binding as B
from tests.rows_common import check_attention, dev, exact_float, random_parents

pytestmark = pytest.mark.gpu

V, KH, D, PAGE, N, SLOTS, BLOCKS, WIDTH, ROT, EPS = 12, 2, 64, 16, 3, 4, 24, 6, 32, 1e-5
I32 = dict(dtype=torch.int32, device="cuda")


class Model:
    """One layer: a token's query, key and value are rows of tables; logits are a product with the attention's result."""

    def __init__(self, H):
        g = torch.Generator().manual_seed(5)
        r = lambda *s: torch.randn(s, generator=g)
        self.H = H
        self.q, self.k, self.v = r(V, H, D).bfloat16(), r(V, KH, D).bfloat16(), r(V, KH, D).bfloat16()
        self.out = (3 * r(H * D, V) / (H * D) ** 0.5).cuda()
        angle = np.arange(WIDTH * PAGE + 8)[:, None] / 100.0 ** (np.arange(ROT // 2) / (ROT // 2))
        self.cos, self.sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
        self.qw, self.kw = [(1 + 0.2 * r(D)).numpy() for _ in range(2)]

    def key(self, token, pos, head):
        return HO.turned(self.k[token, head].float().numpy(), self.cos[pos], self.sin[pos], self.kw, EPS, False)

    def query(self, token, pos, head):
        return HO.turned(self.q[token, head].float().numpy(), self.cos[pos], self.sin[pos], self.qw, EPS, False)

    def cached(self, history):
        """Keys and values [len(history), KH, D] that the cache's codes stand for."""
        out = np.zeros((2, len(history), KH, D))
        for i, t in enumerate(history):
            for h in range(KH):
                for side, x in enumerate((self.key(t, i, h), self.v[t, h].float().numpy())):
                    scales, codes = HO.pack(x)
                    out[side, i, h] = HO.values(scales, HO.packed_bytes(codes))
        return out


def bf16(x):
    return exact_float(torch.from_numpy(np.asarray(x, np.float32)).bfloat16())


class Server:
    def __init__(self, m, M, captured):
        self.m, self.M, self.captured, R = m, M, captured, M + 1
        z = lambda *s: torch.zeros(s, **I32)
        h = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
        byte = lambda *s: torch.full(s, 0xff, dtype=torch.uint8, device="cuda")
        self.cache = [byte(BLOCKS, PAGE, KH, D // 2), byte(BLOCKS, PAGE, KH, D // 2), byte(BLOCKS, PAGE, KH, D // 32), byte(BLOCKS, PAGE, KH, D // 32)]
        self.table, self.ctx, self.added = torch.full((SLOTS, WIDTH), -1, **I32), z(SLOTS), z(SLOTS)
        self.ring, self.ring_state = torch.randperm(BLOCKS, generator=torch.Generator().manual_seed(3)).int().cuda(), torch.tensor([5, BLOCKS], **I32)
        cap = SLOTS * (N + 1)
        self.start, self.slot, self.src, self.pos = z(SLOTS + 1), z(cap), z(cap), z(cap)
        self.tok, self.parent, self.depth, self.count = z(SLOTS, M), z(SLOTS, M), z(SLOTS, M), z(SLOTS)
        self.q, self.q_turned, self.att = h(SLOTS, R, m.H, D), h(SLOTS, R, m.H, D), h(SLOTS, R, m.H, D)
        self.k, self.k_turned, self.v = h(SLOTS, R, KH, D), h(SLOTS, R, KH, D), h(SLOTS, R, KH, D)
        self.logits, self.uniform = torch.zeros((SLOTS, R, V), device="cuda"), torch.zeros((SLOTS, N + 1), device="cuda")
        self.temperature = torch.tensor([0.7, 1.0, 0.0, 1.4], device="cuda")
        self.len, self.out, self.n_out, self.path, self.logp = z(SLOTS), z(SLOTS, N + 1), z(SLOTS), z(SLOTS, N + 1), torch.zeros((SLOTS, N + 1), device="cuda")
        space = lambda n: torch.full((n,), 255, dtype=torch.uint8, device="cuda")
        self.space = space(B.spec_packed_attention_workspace(SLOTS, R, m.H, KH, D))
        self.draws = space(B.spec_verify_sampled_workspace(SLOTS, R, V, torch.float32))
        self.cos, self.sin, self.qw, self.kw = dev(m.cos), dev(m.sin), dev(m.qw), dev(m.kw)
        self.history, self.last = [None] * SLOTS, [0] * SLOTS
        self.graphs = {}

    def run(self, name, call):
        if not self.captured:
            return call()
        if name not in self.graphs:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            self.graphs[name] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graphs[name], stream=side):
                call()
        self.graphs[name].replay()

    def extend(self, add, slot, pos, **kept):
        B.spec_cache_extend(self.ctx, add, self.ctx, self.added, self.table, self.ring, self.ring_state, self.ring_state, PAGE, self.start, slot,
                            pos, **kept)

    def change(self, prompts, ended):
        if ended:
            self.extend(torch.tensor([-(1 << 20) if s in ended else 0 for s in range(SLOTS)], **I32), torch.zeros((0,), **I32), None)
            for s in ended:
                self.history[s] = None
        add = torch.tensor([len(prompts.get(s, [0])) - 1 for s in range(SLOTS)], **I32)
        tokens = [t for s in sorted(prompts) for t in prompts[s][:-1]]
        slot, pos = torch.zeros((len(tokens) + 2,), **I32), torch.zeros((len(tokens) + 2,), **I32)
        self.extend(add, slot, pos)
        rows = torch.tensor(tokens + [0, 0])
        B.spec_packed_append(self.m.k[rows].cuda(), self.m.v[rows].cuda(), slot, *self.cache, pos=pos, cos=self.cos, sin=self.sin, k_weight=self.kw, eps=EPS)
        for s, p in prompts.items():
            self.history[s], self.last[s] = list(p[:-1]), p[-1]

    def step(self, rng):
        m, M, R = self.m, self.M, self.M + 1
        parent = random_parents(rng, SLOTS, M, depth=N)
        tok = rng.integers(0, V, (SLOTS, M))
        depth = np.zeros((SLOTS, M), np.int32)
        for q in range(SLOTS):
            for i in range(M):
                depth[q, i] = 1 + (depth[q, parent[q, i]] if parent[q, i] >= 0 else 0)
        count = np.array([-1 if self.history[s] is None else rng.integers(0, M + 1) for s in range(SLOTS)])
        tokens = np.concatenate([np.array(self.last)[:, None], tok], 1)
        rows = torch.from_numpy(tokens)
        for to, x in ((self.tok, dev(tok)), (self.parent, dev(parent)), (self.depth, dev(depth)), (self.count, dev(count)), (self.q, m.q[rows]),
                      (self.k, m.k[rows]), (self.v, m.v[rows]), (self.uniform, dev(rng.random((SLOTS, N + 1)).astype(np.float32)))):
            to.copy_(x)
        for x in (self.att, self.q_turned, self.k_turned):
            x.fill_(7.0)

        def attend():
            B.spec_rotate_rows(self.q, self.k, self.q_turned, self.k_turned, self.cos, self.sin, ctx_len=self.ctx, node_depth=self.depth, n_nodes=self.count,
                               q_weight=self.qw, k_weight=self.kw, eps=EPS)
            B.spec_packed_attention(self.q_turned, self.k_turned, self.v, *self.cache, self.table, self.ctx, self.parent, self.count, self.att, self.space)
        self.run("attend", attend)
        self.logits.copy_(self.att.flatten(2).float() @ m.out)

        def keep():
            B.spec_verify_sampled(self.logits, self.uniform, self.count, self.len, self.out, self.n_out, self.path, self.draws, self.logp, self.temperature,
                                  node_tok=self.tok, node_parent=self.parent)
            self.extend(self.n_out, self.slot, self.pos, path_row=self.path, seq_rows=R, src_row=self.src)
            B.spec_packed_append(self.k.flatten(0, 1), self.v.flatten(0, 1), self.slot, *self.cache, src_row=self.src, pos=self.pos, cos=self.cos, sin=self.sin,
                                 k_weight=self.kw, eps=EPS)
        self.run("keep", keep)

        # ---- what the oracles say ----
        ctx = np.array([len(x or []) for x in self.history], np.int32)
        most = max(int(ctx.max()), 1)
        k_cache, v_cache = np.zeros((SLOTS, most, KH, D)), np.zeros((SLOTS, most, KH, D))
        q_turned, k_turned = np.zeros((SLOTS, R, m.H, D)), np.zeros((SLOTS, R, KH, D))
        for s in range(SLOTS):
            if self.history[s] is None:
                continue
            k_cache[s, :ctx[s]], v_cache[s, :ctx[s]] = m.cached(self.history[s])
            for r in range(count[s] + 1):
                at = ctx[s] + (depth[s, r - 1] if r else 0)
                q_turned[s, r] = bf16([m.query(tokens[s, r], at, h) for h in range(m.H)])
                k_turned[s, r] = bf16([m.key(tokens[s, r], at, h) for h in range(KH)])
            assert np.array_equal(exact_float(self.q_turned[s, :count[s] + 1]), q_turned[s, :count[s] + 1])
            assert np.array_equal(exact_float(self.k_turned[s, :count[s] + 1]), k_turned[s, :count[s] + 1])
        check_attention(self.att, dict(q=q_turned, k_new=k_turned, v_new=exact_float(self.v), k_cache=k_cache, v_cache=v_cache, table=np.arange(SLOTS)[:, None],
                                       ctx=ctx, parent=parent, n_nodes=count, scale=D ** -0.5), count, torch.full(self.att.shape, 7.0))
        want = SO.verify(self.logits.cpu().numpy(), tok, parent, count, self.temperature.cpu().numpy(), self.uniform.cpu().numpy(), None)
        n, out, path = self.n_out.tolist(), self.out.tolist(), self.path.tolist()
        assert self.added.tolist() == n
        for s, (emitted, kept, _, near) in enumerate(want):
            assert near > 1e-11
            assert out[s][:n[s]] == emitted and path[s][:n[s]] == kept
            if n[s]:
                self.history[s] += [int(tokens[s, r]) for r in kept]
                self.last[s] = emitted[-1]
        return n

    def check_cache(self):
        for s in range(SLOTS):
            if self.history[s]:
                n = len(self.history[s])
                assert int(self.ctx[s]) == n
                at = torch.arange(n, device="cuda")
                slots = (self.table[s][at // PAGE] * PAGE + at % PAGE).int()
                k, v = [torch.zeros((n, KH, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
                B.spec_packed_load(*self.cache, slots, k, v)
                want = self.m.cached(self.history[s])
                assert np.array_equal(exact_float(k), want[0]) and np.array_equal(exact_float(v), want[1])


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("H,M", [(2, 9), (8, 9)])    # up to 32 query rows for a key head, and more
def test_steps_against_the_oracles(H, M, captured):
    rng = np.random.default_rng(6)
    prompt = lambda n: [int(t) for t in rng.integers(0, V, n)]
    s = Server(Model(H), M, captured)
    s.change({0: prompt(20), 1: prompt(1), 2: prompt(33)}, [])
    kept = []
    for step in range(9):
        if step == 3:
            s.change({3: prompt(16)}, [])
        if step == 6:     # two end, and one of their places is taken at once
            s.change({0: prompt(5)}, [0, 2])
        kept += s.step(rng)
    s.check_cache()
    assert 0 in kept and max(kept) >= 2     # (idle places, and steps that kept a node)
    held = [int(x) for q in range(SLOTS) for x in s.table[q, :-(-int(s.ctx[q]) // PAGE)]]
    free = [int(s.ring[(int(s.ring_state[0]) + j) % BLOCKS]) for j in range(int(s.ring_state[1]))]
    assert sorted(held + free) == list(range(BLOCKS))
