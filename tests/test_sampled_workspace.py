"""The workspace of spec_verify_sampled that serves the largest batch and tree of a server serves all smaller ones."""
import pytest
import torch

from paper_2404_19124_amd import binding as B


@pytest.mark.parametrize("V", [1, 7, 5001, 32000, 128256, 300007, 1 << 24, 1 << 30])
def test_the_need_never_falls_as_the_batch_or_the_tree_grows(V):
    """(No GPU needed.)"""
    batches, rows = [1, 2, 3, 4, 5, 8, 10, 16, 31, 64, 500, 4096], [1, 2, 3, 9, 49, 65, 66, 500, 2049, 4097]
    for dtype in (torch.float32, torch.bfloat16):
        need = {(b, R): B.spec_verify_sampled_workspace(b, R, V, dtype) for b in batches for R in rows if b * R <= 1 << 20}
        for (b, R), n in need.items():
            for (c, S), m in need.items():
                assert c > b or S > R or m <= n, ((b, R, n), (c, S, m))


@pytest.mark.gpu
def test_one_buffer_for_every_batch():
    """Of the size for nine sequences, whose rows are taken depth by depth, in calls for fewer, whose rows are taken all at once."""
    from tests.test_gpu_sampled import BF16, Case

    space = Case(9, 40, 70001, 3, BF16, seed=1).args()["workspace"]
    for b in (9, 4, 1, 2, 9):
        c = Case(b, 40, 70001, 3, BF16, seed=b, share=0.8)
        a = c.args()
        own = {k: x.clone() for k, x in a.items() if isinstance(x, torch.Tensor)}
        own["penalties"] = a["penalties"]
        a["workspace"] = space.fill_(255)
        B.spec_verify_sampled(**a)
        B.spec_verify_sampled(**dict(a, **own))
        torch.cuda.synchronize()
        c.check(a)
        for k in ("accept_len", "out_tokens", "n_out", "path_row", "out_logp"):
            assert torch.equal(a[k], own[k]), (b, k)
