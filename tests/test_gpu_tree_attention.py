"""spec_tree_attention against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from paper_2404_19124_amd import binding as B
from oracle import rows_oracle as RO
from tests.rows_common import attention_bound, check_attention, dev, exact_float, random_parents, random_table

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


class Case:
    """Inputs on the device and, exactly the same, in numpy."""

    def __init__(self, H, KH, D, page, M, ctx, dtype="bf16", n_nodes=None, seed=0, depth=7, loud=1.0, extra=3):
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        self.b, self.R, self.H, self.KH, self.D, self.page, self.M = len(ctx), M + 1, H, KH, D, page, M
        self.dtype = DT[dtype]
        need = sum(-(-int(n) // page) for n in ctx)
        width = max([1] + [-(-int(n) // page) for n in ctx]) + 1

        def rand(*shape):
            return torch.randn(shape, generator=gen).to(self.dtype).cuda()

        self.q, self.k_new, self.v_new = rand(self.b, self.R, H, D) * loud, rand(self.b, self.R, KH, D), rand(self.b, self.R, KH, D)
        self.k, self.v = rand(need + extra, page, KH, D), rand(need + extra, page, KH, D)
        self.ctx = np.array(ctx, np.int32)
        self.parent = random_parents(rng, self.b, M, depth)
        self.n_nodes = np.array(n_nodes if n_nodes is not None else [M - (q % 3 if M > 3 else 0) for q in range(self.b)], np.int32)
        self.table = random_table(rng, ctx, page, need + extra, width)
        self.scale = D ** -0.5

    def oracle_args(self):
        f = exact_float
        return dict(q=f(self.q), k_new=f(self.k_new), v_new=f(self.v_new), k_cache=f(self.k), v_cache=f(self.v), table=self.table,
                    ctx=self.ctx, parent=self.parent, n_nodes=self.n_nodes, scale=self.scale)

    def workspace(self):
        # (what lies in a workspace before a call has no meaning)
        n = B.spec_tree_attention_workspace(self.b, self.R, self.H, self.KH, self.D, self.dtype)
        return torch.full((n,), 255, dtype=torch.uint8, device="cuda")

    def run(self, out=None, **kw):
        out = torch.full(self.q.shape, 7.0, dtype=self.dtype, device="cuda") if out is None else out
        a = dict(q=self.q, k_new=self.k_new, v_new=self.v_new, k_cache=self.k, v_cache=self.v, block_table=dev(self.table),
                 ctx_len=dev(self.ctx), node_parent=dev(self.parent), n_nodes=dev(self.n_nodes), out=out, workspace=self.workspace(),
                 scale=self.scale)
        a.update(kw)
        B.spec_tree_attention(**a)
        torch.cuda.synchronize()
        return out

    def check(self, got):
        check_attention(got, self.oracle_args(), self.n_nodes, torch.full(got.shape, 7.0, dtype=self.dtype))


CASES = {
    "chain": dict(H=4, KH=4, D=128, page=16, M=5, ctx=[33, 0, 1, 64, 65]),
    "one_token": dict(H=8, KH=2, D=64, page=16, M=0, ctx=[0, 1, 63, 64, 500]),
    "one_sequence": dict(H=2, KH=2, D=128, page=16, M=36, ctx=[300]),
    "tree_mha": dict(H=3, KH=3, D=128, page=32, M=48, ctx=[0, 17, 128, 255]),
    "tree_gqa": dict(H=16, KH=2, D=128, page=64, M=40, ctx=[129, 70]),
    "tree_mqa_odd": dict(H=7, KH=1, D=80, page=7, M=25, ctx=[100, 3, 64]),
    "wide_tree": dict(H=4, KH=2, D=64, page=16, M=150, ctx=[90, 11]),
    "pages_of_one": dict(H=2, KH=1, D=64, page=1, M=9, ctx=[70, 2]),
    "page_over_tile": dict(H=4, KH=4, D=64, page=200, M=12, ctx=[399, 200, 201]),
    "smallest_head": dict(H=2, KH=2, D=8, page=16, M=12, ctx=[40, 5]),
    "head_of_40": dict(H=2, KH=2, D=40, page=16, M=12, ctx=[40, 5]),
    "head_of_96": dict(H=4, KH=1, D=96, page=16, M=12, ctx=[140, 5]),
    "head_of_192": dict(H=4, KH=1, D=192, page=16, M=12, ctx=[140, 5]),
    "largest_head": dict(H=2, KH=2, D=256, page=16, M=30, ctx=[140, 5]),
    "long": dict(H=2, KH=2, D=64, page=16, M=3, ctx=[3000]),
    "many_sequences": dict(H=2, KH=1, D=64, page=16, M=6, ctx=[(37 * i) % 90 for i in range(150)]),
    "loud_scores": dict(H=4, KH=4, D=64, page=16, M=12, ctx=[200, 31], loud=12.0),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", CASES)
def test_against_the_oracle(name, dtype):
    c = Case(dtype=dtype, seed=len(name), **CASES[name])
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_idle_sequences_and_rows_behind_the_last_are_left_as_they_were(dtype):
    c = Case(4, 2, 64, 16, 20, [50, 60, 70, 0, 5], dtype, n_nodes=[-1, 0, 20, -1, 7])
    # nothing there is read: neither rows behind the last node nor an idle sequence's table
    for q, n in enumerate(c.n_nodes):
        for t in (c.q, c.k_new, c.v_new):
            t[q, n + 1:] = float("nan")
    c.table[0] = -5
    c.parent[0] = 1 << 20
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slots_past_the_length_may_hold_anything(dtype):
    c = Case(4, 2, 128, 48, 20, [50, 100, 1, 0], dtype, seed=3)
    for q, n in enumerate(c.ctx):
        if n % 48:
            last = c.table[q, n // 48]
            c.k[last, n % 48:] = float("nan")
            c.v[last, n % 48:] = float("inf")
    used = set(int(x) for q, n in enumerate(c.ctx) for x in c.table[q, :-(-n // 48)])
    for x in set(range(c.k.shape[0])) - used:
        c.k[x], c.v[x] = float("inf"), float("nan")
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_out_of_range_take_no_part(dtype):
    c = Case(4, 2, 64, 16, 10, [200, 64, 40], dtype, seed=4)
    c.table[0, 2], c.table[0, 7], c.table[0, 12] = -1, c.k.shape[0], 2 ** 31 - 1
    c.table[1, :] = -(2 ** 31)     # nothing of the cache is left
    c.check(c.run())


def test_lengths_and_counts_out_of_range_are_taken_as_the_nearest_within():
    c = Case(4, 2, 64, 16, 10, [32, 48, 16], seed=5)
    wild = c.run(ctx_len=dev(np.array([32, -9, 16], np.int32)), n_nodes=dev(np.array([-7, 10, 1 << 30], np.int32)))
    c.ctx, c.n_nodes = np.array([32, 0, 16], np.int32), np.array([-1, 10, 10], np.int32)
    c.check(wild)


def test_parents_that_do_not_come_before_their_node_end_the_path():
    c = Case(2, 2, 64, 16, 10, [20, 20], seed=6)
    c.parent[0, 4], c.parent[0, 7], c.parent[1, 9] = 4, 9, 2 ** 31 - 1
    c.check(c.run())


def test_a_chain_is_followed_over_eight_nodes():
    c = Case(2, 2, 64, 16, 14, [20], seed=7)
    c.parent[0] = np.arange(14) - 1
    c.n_nodes[:] = 14
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(dtype):
    """Rows out of one product for queries, keys and values, one layer of a cache with heads before slots, an output inside a
    wider buffer."""
    c = Case(6, 2, 64, 16, 12, [100, 31, 0], dtype, seed=8)
    fused = torch.full((c.b, c.R, 6 + 2 + 2, 64 + 8), float("nan"), dtype=c.dtype, device="cuda")
    fused[:, :, :6, :64], fused[:, :, 6:8, :64], fused[:, :, 8:, :64] = c.q, c.k_new, c.v_new
    caches = torch.full((2, 3, c.k.shape[0], 2, 16, 64), float("nan"), dtype=c.dtype, device="cuda")
    caches[0, 1], caches[1, 1] = c.k.transpose(1, 2), c.v.transpose(1, 2)
    wide = torch.full((c.b, c.R, 6, 3, 64), 7.0, dtype=c.dtype, device="cuda")
    c.run(out=wide[:, :, :, 1], q=fused[:, :, :6, :64], k_new=fused[:, :, 6:8, :64], v_new=fused[:, :, 8:, :64],
          k_cache=caches[0, 1].transpose(1, 2), v_cache=caches[1, 1].transpose(1, 2))
    c.check(wide[:, :, :, 1].contiguous())
    assert (wide[:, :, :, 0] == 7).all() and (wide[:, :, :, 2] == 7).all()


def test_one_query_row_for_all_heads_and_a_negative_scale():
    c = Case(4, 1, 64, 16, 5, [80], seed=9)
    c.q = c.q[:, :, :1].expand(-1, -1, 4, -1)
    c.scale = -0.25
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_past_32_bits(dtype):
    """Blocks whose elements lie past 2^31, and past 2^32 bytes."""
    c = Case(2, 1, 64, 16, 6, [40, 33], dtype, seed=10)
    stride = (1 << 29) + 64
    for name in ("k", "v"):
        small = getattr(c, name)
        big = torch.empty(((small.shape[0] - 1) * stride + 16 * 64,), dtype=c.dtype, device="cuda")
        view = big.as_strided((small.shape[0], 16, 1, 64), (stride, 64, 64, 1))
        view.copy_(small)
        setattr(c, name, view)
    assert c.table[:, 0].max() < c.k.shape[0] and (c.k.shape[0] - 1) * stride > 1 << 31
    c.check(c.run())


def test_no_nodes_given():
    c = Case(4, 2, 64, 16, 0, [100, 0, 7], seed=11)
    c.check(c.run(node_parent=None, n_nodes=None))
    c = Case(4, 2, 64, 16, 9, [100, 0, 7], seed=12, n_nodes=[9, 9, 9])
    c.check(c.run(n_nodes=None))


def test_another_stream_and_two_at_once():
    a, b = Case(8, 2, 128, 16, 30, [700, 90, 300], seed=13), Case(8, 2, 128, 16, 30, [500, 400, 0], seed=14)
    wa, wb = a.run(), b.run()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [torch.full(x.q.shape, 7.0, dtype=x.dtype, device="cuda") for x in (a, b)]
    spaces = [a.workspace(), b.workspace()]
    fixed = [dict(block_table=dev(x.table), ctx_len=dev(x.ctx), node_parent=dev(x.parent), n_nodes=dev(x.n_nodes)) for x in (a, b)]
    torch.cuda.synchronize()
    for _ in range(3):
        for x, o, w, f, s in zip((a, b), outs, spaces, fixed, (sa, sb)):
            B.spec_tree_attention(x.q, x.k_new, x.v_new, x.k, x.v, out=o, workspace=w, scale=x.scale, stream=s, **f)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], wa) and torch.equal(outs[1], wb)


def test_captured_and_replayed_with_other_lengths():
    """The same graph serves lengths and trees that change between its replays."""
    cases = [Case(4, 2, 64, 16, 12, ctx, seed=15 + i) for i, ctx in enumerate(([100, 31, 0], [7, 112, 60], [112, 1, 2]))]
    live = cases[0]
    pool = max(c.k.shape[0] for c in cases)
    k, v = (torch.zeros((pool, 16, 2, 64), dtype=live.dtype, device="cuda") for _ in range(2))
    width = max(c.table.shape[1] for c in cases)
    table = torch.zeros((3, width), dtype=torch.int32, device="cuda")
    ctx, parent, count = dev(live.ctx), dev(live.parent), dev(live.n_nodes)
    q, kn, vn, out = live.q.clone(), live.k_new.clone(), live.v_new.clone(), torch.zeros_like(live.q)
    space = live.workspace()

    def call():
        B.spec_tree_attention(q, kn, vn, k, v, table, ctx, parent, count, out, space, live.scale)

    def load(c):
        k[:c.k.shape[0]], v[:c.k.shape[0]] = c.k, c.v
        table[:, :c.table.shape[1]] = dev(c.table)
        for to, x in ((ctx, dev(c.ctx)), (parent, dev(c.parent)), (count, dev(c.n_nodes)), (q, c.q), (kn, c.k_new), (vn, c.v_new)):
            to.copy_(x)
        out.fill_(7.0)

    load(live)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for c in cases + cases[::-1]:
        load(c)
        graph.replay()
        torch.cuda.synchronize()
        c.check(out)


def test_the_same_call_twice_gives_the_same_bits():
    c = Case(16, 4, 128, 16, 40, [900, 20, 333, 64], seed=19)
    first = c.run()
    for _ in range(3):
        assert torch.equal(c.run(), first)


def seen_by(parent, row):
    rows = [0]
    while row > 0 and len(rows) <= 8:
        rows.append(row)
        row = parent[row - 1] + 1
    return rows


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,KH,D,M,ctx", [(2, 2, 64, 9, [5, 0, 40]), (2, 1, 128, 7, [2000, 61]), (8, 2, 128, 20, [300, 3]), (4, 1, 80, 70, [50, 130]),
                                          (8, 1, 128, 30, [700, 64]), (2, 2, 256, 6, [20, 100]), (4, 2, 192, 60, [90])])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(H, KH, D, M, ctx, dtype):
    """Infinities and NaN in a node's values reach the node and those below it, in their elements, and nobody else; NaN in a
    node's keys reaches the same rows whole."""
    c = Case(H, KH, D, 16, M, ctx, dtype, seed=21)
    args = c.oracle_args()
    clean, weighted, products, n_keys = RO.attention(**args)
    bound = attention_bound(clean, weighted, products, n_keys, D, dtype == "bf16")
    marks = {2: (3, float("inf")), 4: (0, float("nan")), 5: (D - 1, float("-inf")), 1: (3, float("-inf"))}   # row: element, value
    for row, (e, x) in marks.items():
        c.v_new[:, row, KH - 1, e] = x
    keys = M if M > 6 else 6
    c.k_new[:, keys, 0, 1] = float("nan")
    got = exact_float(c.run())
    G = H // KH
    for q in range(c.b):
        for r in range(c.n_nodes[q] + 1):
            seen = seen_by(c.parent[q], r)
            for h in range(H):
                want = clean[q, r, h].copy()
                if h // G == KH - 1:
                    for e in (0, 3, D - 1):
                        bad = [x for row, (at, x) in marks.items() if at == e and row in seen]
                        if bad:
                            want[e] = sum(bad)
                if h // G == 0 and keys in seen:
                    want[:] = np.nan
                fine = np.isfinite(want)
                assert np.array_equal(want[~fine], got[q, r, h][~fine], equal_nan=True), (q, r, h)
                off = np.abs(want[fine] - got[q, r, h][fine])
                assert (off <= np.broadcast_to(bound[q, r, h], want.shape)[fine]).all(), (q, r, h)


WIDE = {
    "split_over_workgroups": dict(H=8, KH=1, D=160, page=7, M=40, ctx=[3000, 0, 200]),
    "one_token": dict(H=3, KH=3, D=132, page=16, M=0, ctx=[1, 500, 64, 0]),
    "grouped": dict(H=16, KH=2, D=256, page=64, M=20, ctx=[1000, 70, 129]),
    "many_nodes": dict(H=2, KH=2, D=200, page=16, M=300, ctx=[90]),
    "idle": dict(H=5, KH=1, D=144, page=32, M=9, ctx=[40, 300, 0], n_nodes=[9, -1, 0]),
    "loud": dict(H=4, KH=4, D=256, page=16, M=12, ctx=[200, 31], loud=12.0),
}


@pytest.mark.parametrize("name", WIDE)
def test_wide_float32_heads(name):
    c = Case(dtype="f32", seed=40 + len(name), **WIDE[name])
    c.check(c.run())
    if c.ctx[0] > 2 * c.page:      # blocks that are not there, and parents that are not before their node
        c.table[0, 1], c.table[0, 2] = -1, c.k.shape[0]
        if c.M > 8:
            c.parent[0, 5], c.parent[0, 8] = 7, 2 ** 31 - 1
        c.check(c.run())


def test_wide_float32_heads_captured_and_replayed():
    c = Case(H=6, KH=2, D=192, page=16, M=11, ctx=[700, 33, 0], dtype="f32", seed=51)
    out = torch.full(c.q.shape, 7.0, device="cuda")
    ctx, count = dev(c.ctx), dev(c.n_nodes)
    a = dict(q=c.q, k_new=c.k_new, v_new=c.v_new, k_cache=c.k, v_cache=c.v, block_table=dev(c.table), ctx_len=ctx, node_parent=dev(c.parent),
             n_nodes=count, out=out, workspace=c.workspace(), scale=-c.scale)
    c.scale = -c.scale
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        B.spec_tree_attention(**a)
    for lengths, nodes in (([700, 33, 0], [11, 10, 9]), ([1, 20, 0], [0, -1, 11]), ([600, 0, 0], [11, 11, 0])):
        c.ctx, c.n_nodes = np.array(lengths, np.int32), np.array(nodes, np.int32)
        ctx.copy_(dev(c.ctx))
        count.copy_(dev(c.n_nodes))
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.check(out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shares_that_hold_several_heads(dtype):
    """So many short sequences that a share is several heads' units, in groups of heads that do not divide their number, each of
    several blocks of query rows; some sequences take no part."""
    n_nodes = [-1 if q % 11 == 3 else 8 - q % 4 for q in range(128)]
    c = Case(H=160, KH=5, D=16, page=16, M=8, ctx=[(37 * q) % 150 for q in range(128)], dtype=dtype, seed=61, n_nodes=n_nodes)
    c.check(c.run())
