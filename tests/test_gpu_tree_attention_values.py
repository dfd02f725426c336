"""spec_tree_attention on values and scores at the ends of their ranges."""
import numpy as np
import pytest
import torch

from tests.rows_common import U16, U32, exact_float
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
