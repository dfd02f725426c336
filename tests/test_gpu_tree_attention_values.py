"""spec_tree_attention on values and scores at the ends of their ranges."""
import numpy as np
import pytest
import torch

from paper_2404_19124_amd import binding as B
from tests.rows_common import U16, U32, check_attention, dev, exact_float
from tests.test_gpu_tree_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,KH,D,M,ctx", [(2, 2, 64, 0, [1, 2, 3, 70]), (4, 2, 128, 9, [2, 0, 40, 100]), (8, 1, 128, 30, [1, 200, 3]), (12, 2, 96, 6, [65, 1]),
                                          (2, 1, 256, 25, [3, 64, 500]), (3, 3, 40, 2, [(7 * i) % 23 for i in range(60)])])
def test_values_that_are_all_the_same_come_out_as_they_are(H, KH, D, M, ctx):
    """The weights of a row sum to one, however they are rounded: with the same value v at every key, a row's sum of products, n
    exact ones in float32, and its sum of weights are off by n U32 of themselves each, the quotient and the joins by a few U32
    more: together below 1e-3 of bfloat16's half step, so that v comes out to the bit."""
    c = Case(H, KH, D, 16, M, ctx, "bf16", seed=71, loud=2.0)
    assert (2 * (max(ctx) + M + 64) + 16) * U32 < 0.05 * U16
    v = torch.randn((KH, D), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    c.v[:], c.v_new[:] = v, v
    got = c.run()
    want = v.repeat_interleave(H // KH, 0)
    for q in range(c.b):
        live = got[q, :c.n_nodes[q] + 1]
        assert torch.equal(live, want.expand_as(live)), q


@pytest.mark.parametrize("H,KH,D,M", [(1, 1, 64, 0), (8, 1, 64, 3), (4, 2, 128, 12), (16, 1, 128, 12), (3, 3, 256, 40), (2, 1, 80, 9)])
def test_weights_that_are_all_rounded_the_same_way_do_not_move_the_sum(H, KH, D, M):
    """Of 16 cached keys one and the rows have the largest score, the others a weight of 0.5021, which bfloat16 has as 0.50390625.
    The value, the same at every key, is bfloat16's last one below 2: with the rounded weights over the sum of the exact ones it
    would come out as 2."""
    c = Case(H, KH, D, 16, M, [300, 130], "bf16", seed=72)
    c.q[:], c.k[:], c.k_new[:] = 0, 0, 0
    c.q[..., 0], c.k[:, 1:, :, 0] = 1, -1
    c.scale = -float(np.log(0.5021))
    c.v[:], c.v_new[:] = 1.9921875, 1.9921875
    got = exact_float(c.run())
    for q in range(c.b):
        assert (got[q, :c.n_nodes[q] + 1] == 1.9921875).all(), q


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128, 192, 256])
@pytest.mark.parametrize("H,KH,M", [(1, 1, 0), (8, 2, 3), (4, 1, 40)])
def test_the_largest_values_stay_finite(D, H, KH, M, dtype):
    """A cached key of score 0 and, behind it, rows of score 3: means of values near the type's largest one.  A mean of two or more
    of them is exact to the rounding of the sums (16 U32), of the weights (U16 twice) and of the output."""
    c = Case(H, KH, D, 16, M, [1, 0, 1], dtype, seed=73, depth=1)
    c.q[:], c.k[:], c.k_new[:] = 0, 0, 0
    c.q[..., 0], c.k_new[:, :, :, 0] = 1, 3
    c.scale = 1.0
    sign = torch.where(torch.rand((D,), generator=torch.Generator().manual_seed(6)) < 0.5, -1.0, 1.0).to(c.dtype).cuda()
    c.v[:], c.v_new[:] = 3.0e38 * sign, 2.0e38 * sign
    got = exact_float(c.run())
    a, b = exact_float(c.v[0, 0, 0]), exact_float(c.v_new[0, 0, 0])
    for q in range(c.b):
        for r in range(c.n_nodes[q] + 1):
            seen = 1 + (r > 0)
            w = np.exp(-3.0) * float(c.ctx[q])
            want = (w * a + seen * b) / (w + seen)
            lim = (32 * U32 + (3 * U16 if dtype == "bf16" else 0)) * np.abs(want) * 1.5
            assert bool((np.abs(got[q, r] - want) <= lim).all()), (q, r)


def time_of(case, args):
    """Seconds per call, the best of a few runs of several."""
    best = np.inf
    for _ in range(4):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(3):
            B.spec_tree_attention(**args)
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) / 3e3)
    return best


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,KH,D,M", [(32, 4, 128, 16), (16, 2, 64, 8), (8, 2, 96, 9), (8, 1, 128, 0)])
def test_an_infinity_in_a_cached_value_costs_a_second_pass_at_most(H, KH, D, M, dtype):
    """One request's overflow must not hold up the batch: the workgroups' shares that hold it are gone through twice."""
    c = Case(H, KH, D, 16, M, [3000, 2500, 2000, 2900] * 4, dtype, seed=74)
    # (M == 0: a block that is not there, the other reason for a key that not every row sees)
    c.table[0, 40] = -1
    args = dict(q=c.q, k_new=c.k_new, v_new=c.v_new, k_cache=c.k, v_cache=c.v, block_table=dev(c.table), ctx_len=dev(c.ctx), node_parent=dev(c.parent),
                n_nodes=dev(c.n_nodes), out=torch.full(c.q.shape, 7.0, dtype=c.dtype, device="cuda"), workspace=c.workspace(), scale=c.scale)
    B.spec_tree_attention(**args)
    torch.cuda.synchronize()
    fine, clean = time_of(c, args), args["out"].clone()
    block = int(c.table[0, 100])
    c.v[block, 3, 0, 5] = float("inf")
    B.spec_tree_attention(**args)
    torch.cuda.synchronize()
    odd = time_of(c, args)
    assert odd < 8 * fine + 20e-6, (odd, fine)
    got, G = args["out"].clone(), H // KH
    assert (got[0, :c.n_nodes[0] + 1, :G, 5] == float("inf")).all()
    got[0, :c.n_nodes[0] + 1, :G, 5] = clean[0, :c.n_nodes[0] + 1, :G, 5]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,KH,D,M,ctx", [(2, 2, 40, 3, [100, 20]), (8, 1, 80, 12, [300, 64, 1]), (4, 2, 96, 20, [130]), (2, 1, 192, 6, [70, 9]), (4, 4, 64, 5, [200])])
def test_a_key_of_minus_infinity_has_no_weight(H, KH, D, M, ctx, dtype):
    """Scores of -inf, from the last elements of keys, whatever stands behind them in a tile: the result is that without the key."""
    c = Case(H, KH, D, 16, M, ctx, dtype, seed=75)
    c.q[..., D - 1] = c.q[..., D - 1].abs() + 0.25
    gone = [(q, t) for q, n in enumerate(ctx) for t in range(0, n, 13)]
    for q, t in gone:
        c.k[int(c.table[q, t // 16]), t % 16, :, D - 1] = float("-inf")
    args = c.oracle_args()
    got = c.run()
    # without these keys: the others moved together
    k, v = args["k_cache"], args["v_cache"]
    k2, v2 = np.zeros((sum(ctx) + 1, 1, KH, D)), np.zeros((sum(ctx) + 1, 1, KH, D))
    table, left, at = np.full((len(ctx), max(ctx)), -1, np.int32), [], 0
    for q, n in enumerate(ctx):
        keep = [t for t in range(n) if (q, t) not in gone]
        for i, t in enumerate(keep):
            k2[at, 0], v2[at, 0] = k[c.table[q, t // 16], t % 16], v[c.table[q, t // 16], t % 16]
            table[q, i] = at
            at += 1
        left.append(len(keep))
    args.update(k_cache=k2, v_cache=v2, table=table, ctx=np.array(left, np.int32))
    check_attention(got, args, c.n_nodes, torch.full(got.shape, 7.0, dtype=c.dtype))


@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,KH,D,M,ctx", [(2, 2, 64, 3, [40, 0, 9]), (8, 2, 128, 30, [200, 17]), (16, 1, 128, 20, [70]), (4, 4, 64, 12, [(37 * i) % 150 for i in range(150)]),
                                          (12, 2, 256, 9, [700, 3]), (4, 1, 96, 40, [64, 130, 5]), (2, 1, 160, 12, [90, 2000]), (6, 3, 128, 6, [3000, 1])])
def test_outputs_in_the_place_of_the_queries(H, KH, D, M, ctx, dtype, odd):
    """The same bits as into memory of its own; with infinities, too, which some shares are gone through twice for."""
    c = Case(H, KH, D, 16, M, ctx, dtype, seed=76)
    if odd:
        for q in range(0, c.b, 3):
            c.v_new[q, min(2, M), KH - 1, 3] = float("inf")
            if ctx[q]:
                c.v[int(c.table[q, 0]), 0, 0, 1] = float("-inf")
    want = c.run()
    q = c.q.clone()
    got = c.run(out=q, q=q)
    for s in range(c.b):
        live = int(c.n_nodes[s]) + 1
        assert torch.equal(got[s, :live].nan_to_num(nan=1e30), want[s, :live].nan_to_num(nan=1e30)), s
        assert torch.equal(got[s, live:], c.q[s, live:])
