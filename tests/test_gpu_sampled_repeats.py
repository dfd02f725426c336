"""spec_verify_sampled on drafts that repeat a token along a path (spaces, digits, a word said again): each occurrence counts, in the row's
mass as in its drafted tokens, whatever of it was seen before.  Tolerances are those of the other draws: Case.check."""
import numpy as np
import pytest
import torch

from oracle import sample_oracle as SO
from paper_2404_19124_amd import binding as B
from tests.test_gpu_sampled import BF16, F32, Case

N = 7                                # nodes of the chain
CHAINS = {"alone": "aaaaaaa", "by_twos": "aabaaba", "in_turn": "abababa", "late": "cddaaaa"}
# what is known of the tokens: their bit clear (their counts are then of no account), set, the bits alone, the counts alone, neither
KNOWN = ["clear", "set", "bits", "counts", "paths"]


class Repeats(Case):
    """Per sequence a chain of N nodes with the tokens of `chain`'s letters, and beside each of them a sibling with another token.  Even
    sequences have the repeated token in a whole word of 16, odd ones in a row's tail; every third one has no temperature."""

    def __init__(self, chain, known, b, V, dtype, seed):
        rng = np.random.default_rng(seed)
        M = 2 * N
        self.letters = chain + "z" * N
        self.b, self.M, self.V, self.n, self.dtype, self.n_nodes = b, M, V, N, dtype, None
        chained = np.arange(N) - 1
        self.parent = np.tile(np.concatenate([chained, chained]), (b, 1)).astype(np.int32)
        frequency, presence, repetition = rng.uniform(0.5, 1.5, b), rng.uniform(0, 0.4, b), rng.uniform(1, 1.2, b)
        self.temperature = np.where(np.arange(b) % 3 == 2, 0, rng.uniform(0.8, 1.2, b)).astype(np.float32)
        # so many nodes down for those with a temperature (drafted tokens come first), then anywhere
        self.uniform = np.where(np.arange(N + 1) < 4 + np.arange(b)[:, None] % 4, 0.2, 1.0) * rng.random((b, N + 1))
        self.uniform = self.uniform.astype(np.float32)
        self.tok = np.zeros((b, M), np.int32)
        x = rng.normal(size=(b, M + 1, V)).astype(np.float32)
        words = -(-V // 32)
        bits, counts = np.zeros((b, 32 * words), np.uint32), np.zeros((b, V), np.int32)
        for q in range(b):
            at = 16 * int(rng.integers(0, V // 16)) if q % 2 == 0 else V // 16 * 16
            a = at + int(rng.integers(0, 16 if q % 2 == 0 else V % 16))
            *others, rival = [int(t) for t in rng.choice(V, 6, replace=False) if t != a][:5]
            of = dict(zip("abcdz", [a] + others))
            self.tok[q] = [of[c] for c in self.letters]
            near = [t for t in range(at, min(at + 16, V)) if t not in of.values() and rng.random() < 0.3]
            bits[q, near], counts[q, near] = 1, 3
            told = [of[c] for c in set(chain)]
            counts[q, told] = 2
            bits[q, told] = known == "set"
            for i in range(N):                    # what a row's drafted token is after its penalties; its sibling's
                on_path = chain[:i].count(chain[i])
                c = on_path + (2 if known in ("set", "counts") else 0)
                greedy = self.temperature[q] == 0
                v = 6 if greedy else np.log(V) + 0.5 + 0.3 * rng.normal()
                x[q, i, of[chain[i]]] = (v + frequency[q] * c + presence[q] * (c > 0)) * (repetition[q] if c else 1)
                x[q, i, of["z"]] = 0 if greedy else np.log(V) - 3
                if greedy:                        # the drafted token falls behind another one with its third occurrence
                    x[q, i, rival] = 6 + (0.5 if on_path >= 2 else -0.5) * frequency[q]
        self.logits = torch.from_numpy(x).to(dtype)
        packed = (bits.reshape(b, words, 32) << np.arange(32, dtype=np.uint32)).sum(2).astype(np.uint32).view(np.int32)
        self.pen = {"frequency": frequency.astype(np.float32), "presence": presence.astype(np.float32), "repetition": repetition.astype(np.float32)}
        if known in ("clear", "set", "bits"):
            self.pen["seen"] = packed
        if known in ("clear", "set", "counts"):
            self.pen["counts"] = counts

    def want(self):
        return SO.verify(self.logits.float().numpy(), self.tok, self.parent, None, self.temperature, self.uniform, self.pen)


@pytest.mark.parametrize("chain", CHAINS)
@pytest.mark.parametrize("known", KNOWN)
def test_the_cases_tell_one_occurrence_from_several(chain, known, monkeypatch):
    """(No GPU needed.)  Were a path's token counted once only, the draws or their logarithms would be others by far, with a temperature
    and without."""
    c = Repeats(CHAINS[chain], known, 12, 1003, F32, seed=1)
    want, path_of = c.want(), SO.path_of

    def once(parent, row):
        path = path_of(parent, row)
        return [i for k, i in enumerate(path) if c.letters[i] not in [c.letters[j] for j in path[:k]]]

    monkeypatch.setattr(SO, "path_of", once)
    other = [0, 0]
    for q, (a, b) in enumerate(zip(want, c.want())):
        other[int(c.temperature[q] == 0)] += a[0] != b[0] or float(np.abs(np.array(a[2]) - np.array(b[2])).max()) > 1e-3
    assert min(other) >= 2, other


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("known", KNOWN)
@pytest.mark.parametrize("chain", CHAINS)
def test_few_rows(chain, known, dtype):
    for V in (1003, 4111):
        c = Repeats(CHAINS[chain], known, 12, V, dtype, seed=1)
        c.run(update="counts" in c.pen and "seen" in c.pen)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("known", KNOWN)
def test_depth_by_depth(known, dtype):
    """More than 2^24 logits."""
    c = Repeats(CHAINS["alone" if dtype == F32 else "late"], known, 6, 200003, dtype, seed=2)
    assert c.logits.numel() > 1 << 24
    c.run()


@pytest.mark.gpu
def test_a_repeated_token_comes_as_often_as_its_probability_says():
    """After three of them: 4096 random numbers spread evenly over the row's mass."""
    draws, V, t = 4096, 50, 17
    c = Repeats("aaaaaaa", "clear", 1, V, F32, seed=3)
    c.tok[0, :N], c.tok[0, N:] = t, 30
    c.pen["seen"][:] = 0
    c.logits[:] = 0
    c.logits[:, :, t] = 6
    c.pen.update(frequency=np.array([0.5], np.float32), presence=np.zeros(1, np.float32), repetition=np.ones(1, np.float32))
    c.b, c.temperature = draws, np.ones(draws, np.float32)
    c.logits, c.tok, c.parent = c.logits.expand(draws, -1, -1).contiguous(), np.repeat(c.tok, draws, 0), np.repeat(c.parent, draws, 0)
    c.pen = {k: np.repeat(x, draws, 0) for k, x in c.pen.items()}
    c.uniform = np.zeros((draws, N + 1), np.float32)
    c.uniform[:, 3] = (np.arange(draws) + 0.5) / draws
    c.uniform[:, 4] = 1
    a = c.args()
    B.spec_verify_sampled(**a)
    x = np.zeros(V)
    x[t] = 6 - 3 * 0.5
    p = np.exp(x) / np.exp(x).sum()
    got = np.bincount(a["out_tokens"][:, 3].cpu().numpy(), minlength=V)
    assert got.sum() == draws and (np.abs(got - draws * p) <= 2).all()
