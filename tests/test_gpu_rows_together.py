"""The operators around the base model's forward run together, as a server runs them: prompts are stored, every step attends over
a tree of candidates, verifies its rows under penalties, extends the cache by the kept rows and stores them; sequences end, and
others take their place and their blocks.  With a base model of one layer the emitted tokens are those of decoding token by token."""
import numpy as np
import pytest
import torch

from paper_2404_19124_amd import binding as B

pytestmark = pytest.mark.gpu

V, E, H, KH, D, PAGE, N, C = 61, 32, 4, 2, 16, 4, 3, 6     # vocabulary, width, heads, head, page, draft length, candidates
I32 = dict(dtype=torch.int32, device="cuda")
PENALTY = dict(repetition=1.3, presence=0.2, frequency=0.1)


def _weights():
    g = torch.Generator().manual_seed(2)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)
    return dict(tok=r(V, E), pos=r(80, E), q=r(E, H * D) / E ** 0.5, k=r(E, KH * D) / E ** 0.5, v=r(E, KH * D) / E ** 0.5,
                o=r(H * D, E) / (H * D) ** 0.5, out=r(E, V) / E ** 0.5)


def _decode(w, prompt, steps):
    """Token by token in 64 bits on the host; also the smallest distance of a chosen logit from the next one."""
    seq, counts, margin = list(prompt), np.zeros(V), np.inf
    for _ in range(steps):
        x = w["tok"][seq] + w["pos"][:len(seq)]
        q, k, v = (x[-1:] @ w["q"]).view(H, D), (x @ w["k"]).view(-1, KH, D), (x @ w["v"]).view(-1, KH, D)
        k, v = k.repeat_interleave(H // KH, 1), v.repeat_interleave(H // KH, 1)
        a = torch.einsum("hd,thd->ht", q, k) * D ** -0.5
        o = torch.einsum("ht,thd->hd", torch.softmax(a, -1), v).reshape(1, -1)
        logits = ((x[-1:] + o @ w["o"]) @ w["out"])[0].numpy().copy()
        seen = np.zeros(V, bool)
        seen[seq] = True
        logits = np.where(seen, np.where(logits > 0, logits / PENALTY["repetition"], logits * PENALTY["repetition"]), logits)
        logits = logits - PENALTY["frequency"] * counts - PENALTY["presence"] * (counts > 0)
        best = np.sort(logits)[::-1]
        margin = min(margin, best[0] - best[1])
        seq.append(int(np.argmax(logits)))
        counts[seq[-1]] += 1
    return seq[len(prompt):], margin


class Server:
    def __init__(self, w, slots, captured):
        self.w = {k: x.float().cuda() for k, x in w.items()}
        self.slots, self.captured, R, n_blocks, width = slots, captured, C * N + 1, 40, 16
        z = lambda *s: torch.zeros(s, **I32)
        f = lambda *s: torch.zeros(s, dtype=torch.float32, device="cuda")
        self.k, self.v = f(n_blocks, PAGE, KH, D), f(n_blocks, PAGE, KH, D)
        self.table, self.ctx, self.added = torch.full((slots, width), -1, **I32), z(slots), z(slots)
        self.ring, self.ring_state = torch.randperm(n_blocks, generator=torch.Generator().manual_seed(3)).int().cuda(), torch.tensor([7, n_blocks], **I32)
        self.start, self.slot, self.src = z(slots + 1), z(slots * (N + 1)), z(slots * (N + 1))
        self.last, self.active = z(slots), torch.zeros((slots,), dtype=torch.bool, device="cuda")
        self.cand, self.cand_node = z(slots, C, N), z(slots, C, N)
        self.tok, self.parent, self.depth, self.count = z(slots, R - 1), z(slots, R - 1), z(slots, R - 1), z(slots)
        self.q, self.att = f(slots, R, H, D), f(slots, R, H, D)
        self.kv = f(2, slots, R, KH, D)
        self.space = torch.empty(B.spec_tree_attention_workspace(slots, R, H, KH, D, torch.float32), dtype=torch.uint8, device="cuda")
        self.logits, self.greedy = f(slots, R, V), z(slots, R)
        self.len, self.best, self.out, self.n_out, self.path = z(slots), z(slots), z(slots, N + 1), z(slots), z(slots, N + 1)
        self.pen = {"counts": z(slots, V), "seen": z(slots, 2)}
        self.pen.update({k: torch.full((slots,), x, device="cuda") for k, x in PENALTY.items()})
        self.graphs = {}

    def _run(self, name, call):
        """Captured once and replayed, or called."""
        if not self.captured:
            return call()
        if name not in self.graphs:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            self.graphs[name] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graphs[name], stream=side):
                call()
        self.graphs[name].replay()

    def _extend(self, add, slot, pos=None, **kept):
        B.spec_cache_extend(self.ctx, add, self.ctx, self.added, self.table, self.ring, self.ring_state, self.ring_state, PAGE, self.start, slot,
                            pos, **kept)

    def change(self, prompts, ended):
        """Sequences end, and prompts {slot: tokens} are stored, all but their last tokens."""
        add = torch.zeros((self.slots,), **I32)
        for s in ended:
            add[s] = -(1 << 20)
            self.active[s] = False
        for s, p in prompts.items():
            assert s in ended or not self.active[s]
        if ended:
            self._extend(add, torch.zeros((0,), **I32))
        if prompts:
            add = torch.tensor([len(prompts.get(s, [0])) - 1 for s in range(self.slots)], **I32)
            packed = [t for s in sorted(prompts) for t in prompts[s][:-1]]
            slot, pos = torch.zeros((len(packed) + 3,), **I32), torch.zeros((len(packed) + 3,), **I32)
            self._extend(add, slot, pos)
            assert torch.equal(self.added, add)
            x = self.w["tok"][torch.tensor(packed + [0] * 3, device="cuda")] + self.w["pos"][pos.clamp(min=0).long()]
            B.spec_cache_store((x @ self.w["k"]).view(-1, KH, D), (x @ self.w["v"]).view(-1, KH, D), slot, self.k, self.v)
            for s, p in prompts.items():
                self.last[s], self.active[s] = p[-1], True
                self.pen["counts"][s] = 0
                bits = np.zeros(64, np.uint8)
                bits[list(p)] = 1
                self.pen["seen"][s] = torch.from_numpy(np.packbits(bits, bitorder="little").view(np.int32).copy()).cuda()

    def step(self, cand):
        self.cand.copy_(torch.tensor(cand, dtype=torch.int32))
        B.spec_tree_metadata(self.cand, self.tok, self.parent, self.depth, self.count, self.cand_node)
        self.count.copy_(torch.where(self.active, self.count, torch.full_like(self.count, -1)))
        live = torch.arange(C * N, device="cuda")[None] < self.count[:, None]
        tokens = torch.cat([self.last[:, None], torch.where(live, self.tok, 0)], 1).long()
        place = self.ctx[:, None] + torch.cat([torch.zeros_like(self.last)[:, None], torch.where(live, self.depth, 0)], 1)
        x = self.w["tok"][tokens] + self.w["pos"][place.long()]
        self.q.copy_((x @ self.w["q"]).view(self.q.shape))
        self.kv[0].copy_((x @ self.w["k"]).view(self.kv[0].shape))
        self.kv[1].copy_((x @ self.w["v"]).view(self.kv[0].shape))
        self._run("attention", lambda: B.spec_tree_attention(self.q, self.kv[0], self.kv[1], self.k, self.v, self.table, self.ctx, self.parent,
                                                             self.count, self.att, self.space))
        self.logits.copy_((x + self.att.flatten(2) @ self.w["o"]) @ self.w["out"])

        def rest():
            B.spec_verify_tree(self.logits, self.cand, self.cand_node, self.count, self.greedy, self.len, self.best, self.out, self.n_out,
                               self.path, penalties=self.pen, node_tok=self.tok, node_parent=self.parent, update=True)
            self._extend(self.n_out, self.slot, path_row=self.path, seq_rows=C * N + 1, src_row=self.src)
            B.spec_cache_store(self.kv[0].flatten(0, 1), self.kv[1].flatten(0, 1), self.slot, self.k, self.v, self.src)
        self._run("rest", rest)
        n, out = self.n_out.tolist(), self.out.tolist()
        assert self.added.tolist() == n
        for s in range(self.slots):
            if n[s]:
                self.last[s] = out[s][n[s] - 1]
        return [out[s][:n[s]] for s in range(self.slots)]


@pytest.mark.parametrize("none_right", [False, True])
@pytest.mark.parametrize("captured", [False, True])
def test_steps_emit_what_decoding_token_by_token_does(captured, none_right):
    w, rng = _weights(), np.random.default_rng(4)
    prompts = [[int(t) for t in rng.integers(0, V, n)] for n in (9, 1, 14, 4, 6, 2)]
    want = []
    for p in prompts:
        tokens, margin = _decode(w, p, 14 * (N + 1))
        # a float32 product of 32 terms is off by at most 32 * 2^-24 * (sum of magnitudes), and those sums stay below 32 here: 6e-5 per
        # product at worst; the embeddings' sum reaches the logits through one of them, the attention through two more
        assert margin > 2e-4
        want.append(tokens)
    s = Server(w, 4, captured)
    of, got = {0: 0, 1: 1, 2: 2}, {i: [] for i in range(6)}     # slot -> prompt
    s.change({slot: prompts[i] for slot, i in of.items()}, [])
    kept = []
    for step in range(14):
        if step == 4:     # a fourth sequence
            of[3] = 3
            s.change({3: prompts[3]}, [])
        if step == 7:     # two end, and one of their places is taken at once
            s.change({1: prompts[4]}, [0, 1])
            del of[0]
            of[1] = 4
        if step == 9:
            of[0] = 5
            s.change({0: prompts[5]}, [])
        cand = rng.integers(0, V, (4, C, N))
        for slot, i in of.items():
            true = want[i][len(got[i]):len(got[i]) + N]
            for c in range(C):      # candidates that are right for 0 to N tokens
                right = int(rng.integers(0, N + 1)) if step % 3 else c % 2
                cand[slot, c, :right] = true[:right]
            if none_right:
                cand[slot, :, 0] = (true[0] + 1) % V
        for slot, tokens in enumerate(s.step(cand.tolist())):
            if slot not in of:
                assert tokens == []
                continue
            i = of[slot]
            best = max(sum(np.cumprod(cand[slot, c] == want[i][len(got[i]):len(got[i]) + N])) for c in range(C))
            assert len(tokens) == best + 1
            got[i] += tokens
            assert got[i] == want[i][:len(got[i])]
            kept.append(len(tokens))
        held = [int(x) for slot in range(4) for x in s.table[slot, :-(-int(s.ctx[slot]) // PAGE)]]
        free = [int(s.ring[(int(s.ring_state[0]) + j) % 40]) for j in range(int(s.ring_state[1]))]
        assert sorted(held + free) == list(range(40))
    assert set(kept) == {1} if none_right else max(kept) == N + 1 and min(kept) < N
