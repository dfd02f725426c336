"""Trees, caches and error bounds of the tests of the operators on a tree's rows."""
import numpy as np
import torch

from oracle import rows_oracle as RO

U32 = 2.0 ** -24
U16 = 2.0 ** -8    # bfloat16: half a step, relative to the value


def random_parents(rng, b, M, depth=7):
    """Parents of M nodes each, a parent before its node, chains of up to `depth` nodes."""
    parent = np.full((b, M), -1, np.int32)
    for q in range(b):
        level = []
        for i in range(M):
            up = int(rng.integers(-1, i)) if i else -1
            if up >= 0 and level[up] >= depth:
                up = -1
            parent[q, i] = up
            level.append(1 if up < 0 else level[up] + 1)
    return parent


def random_table(rng, ctx, page, n_blocks, width):
    """Tables over disjoint blocks in any order; entries behind the last block are out of range."""
    order = rng.permutation(n_blocks)
    table, at = np.full((len(ctx), width), 1 << 30, np.int32), 0
    for q, n in enumerate(ctx):
        need = -(-int(n) // page)
        table[q, :need] = order[at:at + need]
        at += need
    return table


def attention_bound(out, weighted, products, keys, D, bf16):
    """Largest error of a result in float32 arithmetic on exact inputs, per element.

    A score is a sum of D products in some order: off by (D + 3) U32 times the sum of their sizes.  The exponent's argument (a
    product, a difference of numbers up to `products`) is off by 4 U32 products, the exponential by 8 U32: a weight is off by e
    relative to its size, a weight over the sum of weights by 2 e.  Sums over the keys, and the joins of their parts, add
    (keys + 64) U32 twice.  Where weights are rounded to bfloat16 each is off by U16 more, and the result is rounded once."""
    e = (D + 3) * U32 * products + 4 * U32 * products + 8 * U32
    bound = (2 * e + 2 * (keys + 64) * U32) * weighted + U32 * np.abs(out)
    if bf16:
        bound = bound * (1 + U16) + U16 * weighted + U16 * np.abs(out)
    return bound * 1.01 + 1e-37


def dev(x, dtype=None):
    t = torch.as_tensor(np.ascontiguousarray(x))
    return t.to(device="cuda", dtype=dtype) if dtype is not None else t.cuda()


def exact_float(t):
    """Values of a tensor as float64."""
    return t.detach().cpu().double().numpy()


def check_attention(got, args, n_nodes, before):
    """got [b, R, H, D] against the oracle on numpy args; rows that do not exist as they were `before`."""
    out, weighted, products, keys = RO.attention(**args)
    D, bf16 = out.shape[3], got.dtype == torch.bfloat16
    bound = attention_bound(out, weighted, products, keys, D, bf16)
    g, was = exact_float(got), exact_float(before)
    for q in range(out.shape[0]):
        live = int(n_nodes[q]) + 1
        off = np.abs(g[q, :live] - out[q, :live])
        assert (off <= bound[q, :live]).all(), (q, float((off / bound[q, :live]).max()))
        assert np.array_equal(g[q, live:], was[q, live:]), "rows behind sequence %d were written" % q
