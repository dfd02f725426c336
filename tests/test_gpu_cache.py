"""spec_cache_extend and spec_cache_store: every word against the oracle."""
import numpy as np
import pytest
import torch

from oracle import rows_oracle as RO
from paper_2404_19124_amd import binding as B
from tests.rows_common import dev

pytestmark = pytest.mark.gpu


class Server:
    """A batch of sequences that hold disjoint blocks, the rest of the blocks in the ring."""

    def __init__(self, rng, b, page, ctx, n_blocks, width):
        self.page, self.ctx = page, np.array(ctx, np.int32)
        order, at = rng.permutation(n_blocks).astype(np.int32), 0
        self.table = np.full((b, width), -1, np.int32)
        for q, n in enumerate(ctx):
            need = -(-int(n) // page)
            self.table[q, :need] = order[at:at + need]
            at += need
        head = int(rng.integers(n_blocks))
        self.ring = np.full((n_blocks,), -7, np.int32)
        self.ring[(head + np.arange(n_blocks - at)) % n_blocks] = order[at:]
        self.state = [head, n_blocks - at]

    def step(self, add, cap, path=None, seq_rows=0, in_place=False):
        """One call on the device, checked word by word; then the oracle's answer is the new state."""
        b = len(self.ctx)
        want = RO.extend(self.ctx, add, self.table, self.ring, self.state, self.page, cap, path, seq_rows)
        ctx, state = dev(self.ctx), dev(np.array(self.state, np.int32))
        got = dict(new_len=ctx if in_place else torch.full((b,), -9, dtype=torch.int32, device="cuda"),
                   added=torch.full((b,), -9, dtype=torch.int32, device="cuda"), block_table=dev(self.table), ring=dev(self.ring),
                   ring_state_new=state if in_place else torch.full((2,), -9, dtype=torch.int32, device="cuda"),
                   row_start=torch.full((b + 1,), -9, dtype=torch.int32, device="cuda"))
        for k in ("slot", "pos") + (("src_row",) if path is not None else ()):
            got[k] = torch.full((cap,), -9, dtype=torch.int32, device="cuda")
        B.spec_cache_extend(ctx, dev(np.array(add, np.int32)), got["new_len"], got["added"], got["block_table"], got["ring"], state,
                            got["ring_state_new"], self.page, got["row_start"], got["slot"], got["pos"],
                            None if path is None else dev(np.array(path, np.int32)), seq_rows, got.get("src_row"))
        torch.cuda.synchronize()
        for k, w in want.items():
            assert np.array_equal(got[k].cpu().numpy(), np.array(w, np.int32)), k
        self.ctx, self.table, self.ring = np.array(want["new_len"], np.int32), want["block_table"], want["ring"]
        self.state = want["ring_state_new"]
        return want


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("b,page,n_blocks,width", [(1, 1, 40, 30), (7, 16, 60, 12), (64, 3, 700, 40), (300, 16, 2000, 9), (1500, 4, 6000, 8)])
def test_a_run_of_steps(b, page, n_blocks, width, in_place):
    """Growth, rest, trims, ends and shortage mixed; no block is lost and none is held twice."""
    rng = np.random.default_rng(b)
    s = Server(rng, b, page, [0] * b, n_blocks, width)
    for _ in range(12):
        add = [int(rng.choice([0, 1, 2, 3, page, 2 * page + 1, -1, -page, -10 ** 6])) for _ in range(b)]
        s.step(add, cap=int(rng.choice([2 * b + 1, 3 * (page + 2) * b])), in_place=in_place)
        held = [x for q in range(b) for x in s.table[q, :-(-int(s.ctx[q]) // page)]]
        free = [s.ring[(s.state[0] + i) % n_blocks] for i in range(s.state[1])]
        assert sorted(held + free) == list(range(n_blocks))


def test_prompts():
    rng = np.random.default_rng(1)
    s = Server(rng, 5, 16, [0, 300, 0, 17, 0], 2000, 400)
    w = s.step([5000, -300, 1, 0, 6400], cap=12000)
    assert w["added"] == [5000, -300, 1, 0, 6400]
    s.step([16, 16, 16, 16, 1], cap=100)    # the last one has no room in its table, and holds up nobody


def test_requests_are_served_in_order_until_one_does_not_fit():
    rng = np.random.default_rng(2)
    s = Server(rng, 6, 4, [0] * 6, 8, 20)
    w = s.step([8, 0, 12, 16, 1, 0], cap=100)
    assert w["added"] == [8, 0, 12, 0, 0, 0] and w["ring_state_new"][1] == 3
    w = s.step([0, 0, 0, 3, 4, 1], cap=6)      # rows run out
    assert w["added"] == [0, 0, 0, 3, 0, 0]
    w = s.step([-8, 0, 0, 0, 12, 0], cap=100)  # what is given back is handed out by the next call
    assert w["added"] == [-8, 0, 0, 0, 0, 0]
    assert s.step([0, 0, 0, 0, 12, 0], cap=100)["added"] == [0, 0, 0, 0, 12, 0]


def test_kept_rows():
    rng = np.random.default_rng(3)
    s = Server(rng, 5, 16, [15, 16, 0, 31, 40], 40, 10)
    path = [[0, 3, 7, 9], [0, -1, -1, -1], [0, 1, 2, 99], [0, 5, -1, -1], [0, 2, 6, -1]]
    w = s.step([4, 1, 4, 2, 0], cap=20, path=path, seq_rows=10)
    assert w["src_row"][:5] == [0, 3, 7, 9, 10] and w["src_row"][8] == -1
    s.step([3, 1, 5, 2, 0], cap=10, path=[r[:2] for r in path], seq_rows=10)   # paths shorter than what is added


def test_no_rows_at_all():
    s = Server(np.random.default_rng(4), 3, 16, [5, 40, 0], 9, 6)
    assert s.step([1, -20, 3], cap=0)["added"] == [0, -20, 0]


def test_state_out_of_range_reads_and_writes_nothing_outside():
    """Corrupted lengths, ring states and tables give answers without meaning, within the buffers."""
    b, page, n_blocks, width, cap = 4, 16, 10, 6, 50
    guard = torch.full((3, 400), -77, dtype=torch.int32, device="cuda")
    table, ring, slot = guard[0, 100:100 + b * width].view(b, width), guard[1, 100:100 + n_blocks], guard[2, 100:100 + cap]
    for state, ctx in (([-5, 1 << 30], [-3, 1 << 30, 20, 7]), ([1 << 30, -5], [96, 95, 97, 0]), ([3, 10], [2 ** 31 - 1, -2 ** 31, 0, 1])):
        table.fill_(-(2 ** 31)), ring.fill_(2 ** 31 - 1)
        out = [torch.zeros((n,), dtype=torch.int32, device="cuda") for n in (b, b, 2, b + 1)]
        B.spec_cache_extend(dev(np.array(ctx, np.int32)), dev(np.array([5, -2 ** 31, 2 ** 31 - 1, 3], np.int32)), out[0], out[1], table, ring,
                            dev(np.array(state, np.int32)), out[2], page, out[3], slot)
        torch.cuda.synchronize()
        assert (slot == -1).all()
    for g, n in zip(guard, (b * width, n_blocks, cap)):
        assert (g[:100] == -77).all() and (g[100 + n:] == -77).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("L,KH,D,rows,page", [(1, 1, 8, 1, 1), (3, 2, 64, 30, 16), (2, 5, 40, 17, 7), (1, 8, 256, 300, 64)])
def test_store(dtype, L, KH, D, rows, page):
    rng, gen = np.random.default_rng(rows), torch.Generator().manual_seed(rows)
    n_blocks = -(-2 * rows // page) + 1
    k, v, kc, vc = (torch.randn(s, generator=gen).to(dtype).cuda() for s in
                    ((L, rows, KH, D), (L, rows, KH, D), (L, n_blocks, page, KH, D), (L, n_blocks, page, KH, D)))
    slot = rng.permutation(n_blocks * page)[:rows].astype(np.int32)
    if rows > 4:
        slot[1], slot[3] = -1, n_blocks * page
    for src in (None, rng.integers(0, rows, rows).astype(np.int32)):
        if src is not None and rows > 4:
            src[0], src[2] = -1, rows
        want = [RO.store(a.float().cpu().numpy(), slot, c.float().cpu().numpy(), src) for a, c in ((k, kc), (v, vc))]
        B.spec_cache_store(k, v, dev(slot), kc, vc, None if src is None else dev(src))
        torch.cuda.synchronize()
        for w, c in zip(want, (kc, vc)):
            assert np.array_equal(c.float().cpu().numpy(), w)
    if L == 1:   # without the dimension of layers
        kc2, vc2 = torch.zeros_like(kc[0]), torch.zeros_like(vc[0])
        B.spec_cache_store(k[0], v[0], dev(slot), kc2, vc2)
        want = RO.store(k.float().cpu().numpy(), slot, torch.zeros(kc.shape).numpy())[0]
        assert np.array_equal(kc2.float().cpu().numpy(), want)


def test_store_strides():
    """Keys and values out of one product, into one cache tensor that holds both, heads before slots."""
    gen = torch.Generator().manual_seed(0)
    L, rows, KH, D, n_blocks, page = 3, 11, 4, 64, 5, 16
    fused = torch.randn((rows, L, 2 * KH, D), generator=gen).cuda()
    cache = torch.full((n_blocks, L, 2, KH, page, D), 3.0, device="cuda")
    k, v = fused[:, :, :KH].transpose(0, 1), fused[:, :, KH:].transpose(0, 1)
    kc, vc = (cache[:, :, i].permute(1, 0, 3, 2, 4) for i in range(2))
    slot = np.arange(70, 70 - rows, -1).astype(np.int32)
    want = [RO.store(a.cpu().numpy(), slot, c.cpu().numpy()) for a, c in ((k, kc), (v, vc))]
    B.spec_cache_store(k, v, dev(slot), kc, vc)
    assert np.array_equal(kc.cpu().numpy(), want[0]) and np.array_equal(vc.cpu().numpy(), want[1])


def test_store_past_32_bits():
    stride, page, D = (1 << 29) + 64, 4, 64
    caches = [torch.zeros((8 * stride + 4096,), dtype=torch.bfloat16, device="cuda").as_strided((9, page, 1, D), (stride, D, D, 1)) for _ in range(2)]
    k, v = torch.randn((3, 1, D), device="cuda").bfloat16(), torch.randn((3, 1, D), device="cuda").bfloat16()
    # (the last block would reach past the buffer: its slots are not used)
    B.spec_cache_store(k, v, dev(np.array([7 * page + 3, 1, 6 * page], np.int32)), *caches)
    for c, x in zip(caches, (k, v)):
        assert torch.equal(c[7, 3], x[0]) and torch.equal(c[0, 1], x[1]) and torch.equal(c[6, 0], x[2])
        assert c[7].count_nonzero() == x[0].count_nonzero()


def test_nothing_to_store():
    kc = torch.zeros((2, 4, 1, 8), device="cuda")
    none = torch.zeros((0,), dtype=torch.int32, device="cuda")
    B.spec_cache_store(torch.zeros((0, 1, 8), device="cuda"), torch.zeros((0, 1, 8), device="cuda"), none, kc, kc.clone())
    B.spec_cache_store(torch.ones((3, 1, 8), device="cuda"), torch.ones((3, 1, 8), device="cuda"), none, kc, kc.clone())
    B.spec_cache_store(torch.zeros((0, 1, 8), device="cuda"), torch.zeros((0, 1, 8), device="cuda"),
                       torch.zeros((2,), dtype=torch.int32, device="cuda"), kc, kc.clone(), torch.zeros((2,), dtype=torch.int32, device="cuda"))
    assert (kc == 0).all()


@pytest.mark.parametrize("b,cap", [(1, 4096), (1, 4097), (1024, 4096), (1024, 4097), (1025, 4096), (1023, 500)])
def test_where_one_kernel_becomes_two(b, cap):
    """Up to 1024 sequences and 4096 entries of the slot map are one kernel, more are two."""
    rng = np.random.default_rng(b + cap)
    s = Server(rng, b, 16, [0] * b, 1500, 700)
    s.step([1 + q % 7 for q in range(b)], cap=cap)
    add = [int(x) for x in rng.integers(-5, 20, b)]
    add[b // 2] = 6000                      # more than the blocks or the slot map, or just within
    s.step(add, cap=cap)
    add = [-3] * b
    add[b // 2] = 9000 if b == 1 else -10 ** 6
    s.step(add, cap=cap, in_place=True)
    s.step([1] * b, cap=cap, path=[[4, 2]] * b, seq_rows=5)


@pytest.mark.parametrize("b", [1025, 3000, 65535])
def test_large_batches(b):
    """Growth, ends and shortage in batches of which a workgroup takes several sequences."""
    rng = np.random.default_rng(b)
    s = Server(rng, b, 4, [0] * b, 3 * b, 6)
    for share in (0.9, 0.5, 0.2):
        add = np.where(rng.random(b) < share, rng.integers(0, 9, b), np.where(rng.random(b) < 0.5, -10 ** 6, -rng.integers(0, 5, b)))
        s.step(add.tolist(), cap=max(5000, 6 * b), path=rng.integers(0, 4, (b, 3)).tolist(), seq_rows=4)


def test_the_largest_batch_takes_a_time_like_its_size():
    """65535 sequences against 2047: a hundred times at most (32 times the sequences; all of them summed up per sequence is a thousand
    times the work, and took two thousand times as long)."""
    i32 = dict(dtype=torch.int32, device="cuda")
    took = []
    for b in (2047, 65535):
        add, z = torch.full((b,), 3, **i32), lambda *s: torch.zeros(s, **i32)
        args = (z(b), add, z(b), z(b), z(b, 2), torch.arange(b, **i32), torch.tensor([0, b], **i32), z(2), 16, z(b + 1), z(4 * b))
        best = np.inf
        for _ in range(5):
            t = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
            t[0].record()
            B.spec_cache_extend(*args)
            t[1].record()
            torch.cuda.synchronize()
            best = min(best, t[0].elapsed_time(t[1]))
        assert args[3].eq(3).all()
        took.append(best)
    assert took[1] < 100 * took[0], took
