"""Norms and rotation of heads, the append to a cache of the same type and to one of four bits, and the load from that, against the
definitions.  Their roundings are part of the definitions, so results are compared bit by bit with those of numpy's float32; the mean
in a norm is a 64-bit sum, whose order moves it by 1e-16 of itself and the float32 factor with a chance of about 1e-8 per head.  They are
compared with 64 bits too."""
import numpy as np
import pytest
import torch

from oracle import heads_oracle as HO
from paper_2404_19124_amd import binding as B
from tests.rows_common import U16, U32, dev, exact_float

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


def table(rot, n, rng):
    a = rng.normal(size=(n, rot // 2)) * 20
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def rounded(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype)


def floats(t):
    return t.detach().float().cpu().numpy()


def same(a, b):
    """bit by bit, but for the sign of zeros and which NaN"""
    a, b = a.cpu(), b.cpu()
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


def heads(rng, shape, dtype):
    loud = 1 + 5 * (rng.random(shape[-1]) < 0.1)
    return rounded((rng.normal(size=shape) * loud).astype(np.float32), dtype).cuda()


def expected(x, pos, cs, weight, pairs, before):
    """x [b, R, H, D], pos [b, R] with None where there is no row: (what the definition gives, largest error against 64 bits in shares
    of what float32 and the last rounding may be off)"""
    xs, out = floats(x), before.cpu().clone()
    want64, bound = np.zeros(xs.shape), np.zeros(xs.shape)
    u = U16 if x.dtype == BF16 else U32
    for i in np.ndindex(xs.shape[:3]):
        at = pos[i[0]][i[1]]
        if at is None or (cs is not None and not 0 <= at < len(cs[0])):
            continue
        c, s = (cs[0][at], cs[1][at]) if cs is not None else (None, None)
        out[i] = rounded(HO.turned(xs[i], c, s, weight, EPS, pairs), x.dtype)
        want64[i], size = HO.turned64(xs[i], c, s, weight, EPS, pairs)
        # the factor, two products of the norm, a product and a sum of the rotation, the last rounding
        bound[i] = 5.1 * U32 * size + 1.01 * u * np.abs(want64[i]) + 1e-30
        assert (np.abs(exact_float(out[i]) - want64[i]) <= bound[i]).all()
    return out


ROTATE = [  # dtype, heads, key heads, D, rot, pairs, norms, batch, M
    (BF16, 4, 2, 128, 128, False, (True, True), 2, 5), (BF16, 3, 1, 128, 64, True, (False, False), 1, 0), (F32, 4, 4, 80, 48, False, (True, False), 3, 4),
    (F32, 2, 1, 256, 256, True, (False, True), 1, 3), (BF16, 5, 5, 64, 16, False, (False, True), 2, 9), (BF16, 1, 1, 256, 256, False, (True, True), 1, 2),
    (BF16, 7, 1, 80, 80, True, (True, True), 5, 1), (F32, 6, 2, 8, 8, False, (False, False), 2, 3), (BF16, 70, 9, 16, 16, False, (True, True), 3, 7),
    (BF16, 4, 2, 48, 0, False, (True, True), 2, 3), (F32, 3, 3, 252, 248, True, (True, True), 1, 1), (BF16, 2, 1, 256, 32, False, (True, True), 2, 2)]


@pytest.mark.parametrize("dtype,H,KH,D,rot,pairs,norms,b,M", ROTATE)
@pytest.mark.parametrize("by_tree", [True, False])
def test_rotate(dtype, H, KH, D, rot, pairs, norms, b, M, by_tree):
    rng = np.random.default_rng(H * 1000 + D + M)
    R, n_pos = M + 1, 40
    # (one product's heads side by side, as a model's projection gives them)
    both = heads(rng, (b, R, H + 2 * KH, D), dtype)
    q, k = both[:, :, :H], both[:, :, H:H + KH]
    cs = table(rot, n_pos, rng) if rot else None
    wq, wk = ((1 + 0.2 * rng.normal(size=D)).astype(np.float32) if n else None for n in norms)
    if by_tree:
        ctx, depth = rng.integers(0, n_pos, b), rng.integers(1, 9, (b, M))
        nodes = rng.integers(-1, M + 1, b)
        nodes[0] = M
        pos = [[None if r > nodes[s] else int(ctx[s]) + (int(depth[s][r - 1]) if r else 0) for r in range(R)] for s in range(b)]
        where = dict(ctx_len=dev(ctx, torch.int32), node_depth=dev(depth, torch.int32), n_nodes=dev(nodes, torch.int32))
    else:
        at = rng.integers(-2, n_pos + 2, (b, R))
        pos = [[None if x < 0 else int(x) for x in row] for row in at]
        where = dict(pos=dev(at, torch.int32))
    out = [heads(rng, (b, R, R + 2, n, D), dtype)[:, :, 1] for n in (H, KH)]
    before = [x.clone() for x in out]
    cos, sin = (dev(x) for x in cs) if rot else (None, None)
    more = dict(q_weight=None if wq is None else dev(wq), k_weight=None if wk is None else dev(wk), eps=EPS, pairs=pairs, **where)
    B.spec_rotate_rows(q, k, out[0], out[1], cos, sin, **more)
    want = [expected(x, pos, cs, w, pairs, y) for x, w, y in ((q, wq, before[0]), (k, wk, before[1]))]
    assert same(out[0], want[0]) and same(out[1], want[1])
    # queries alone, then both in place; rows that do not exist keep what they hold
    alone = before[0].clone()
    B.spec_rotate_rows(q, None, alone, None, cos, sin, **dict(more, k_weight=None))
    assert torch.equal(alone, out[0])
    original = both.clone()
    B.spec_rotate_rows(q, k, q, k, cos, sin, **more)
    for x, y, w, done in ((q, original[:, :, :H], wq, out[0]), (k, original[:, :, H:H + KH], wk, out[1])):
        assert same(x, expected(y, pos, cs, w, pairs, y))
    assert torch.equal(both[:, :, H + KH:], original[:, :, H + KH:])


def test_rotate_values_that_are_not_finite_stay_in_their_pairs():
    rng = np.random.default_rng(9)
    cs = table(64, 3, rng)
    for bad in (np.inf, np.nan, -np.inf):
        x = heads(rng, (1, 3, 2, 64), BF16)
        x[0, 1, 0, 5] = bad
        out = torch.zeros_like(x)
        B.spec_rotate_rows(x, None, out, None, dev(cs[0]), dev(cs[1]), pos=dev([[0, 1, 2]], torch.int32))
        assert same(out, expected_nan(x, cs))
        gone = ~out.isfinite().cpu()
        assert sorted(map(tuple, gone.nonzero().tolist())) == [(0, 1, 0, 5), (0, 1, 0, 37)]


def expected_nan(x, cs):
    xs, out = floats(x), x.cpu().clone()
    with np.errstate(invalid="ignore"):
        for i in np.ndindex(xs.shape[:3]):
            out[i] = rounded(HO.turned(xs[i], cs[0][i[1]], cs[1][i[1]], None, EPS, False), x.dtype)
    return out


def test_rotate_captured_and_on_another_stream():
    rng = np.random.default_rng(10)
    cs = [dev(x) for x in table(128, 900, rng)]
    q, k, w = heads(rng, (3, 4, 8, 128), BF16), heads(rng, (3, 4, 2, 128), BF16), dev(np.ones(128, np.float32))
    ctx, depth, nodes = dev([5, 800, 0], torch.int32), dev(rng.integers(1, 4, (3, 3)), torch.int32), dev([3, 1, 2], torch.int32)
    out = [torch.zeros_like(q), torch.zeros_like(k)]
    args = (q, k, *out, *cs)
    more = dict(ctx_len=ctx, node_depth=depth, n_nodes=nodes, q_weight=w, k_weight=w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.spec_rotate_rows(*args, stream=side, **more)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.spec_rotate_rows(*args, **more)
    for turn in range(4):
        q.copy_(heads(rng, (3, 4, 8, 128), BF16))
        ctx.copy_(dev([7 * turn, 31, 2], torch.int32))
        want = [torch.zeros_like(q), torch.zeros_like(k)]
        B.spec_rotate_rows(q, k, *want, *cs, **more)
        out[0].zero_(), out[1].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])


# ---- append -------------------------------------------------------------------------------------------------------

def entries(rng, n_slots, rows, count, n_pos):
    slot = rng.permutation(n_slots)[:count].astype(np.int64)
    slot[rng.random(count) < 0.15] = -1
    if count > 3:
        slot[1], slot[2] = n_slots, 1 << 30
    return slot, rng.integers(-1, rows + 1, count), rng.integers(-1, n_pos + 1, count)


APPEND = [  # dtype, layers, heads, D, rot, pairs, norm, blocks, page, rows, count, own rows
    (BF16, 1, 4, 128, 128, False, True, 5, 16, 30, 30, False), (BF16, 3, 2, 64, 32, True, True, 4, 7, 20, 11, True), (F32, 2, 3, 80, 80, False, False, 3, 5, 9, 14, True),
    (F32, 1, 1, 256, 64, True, True, 2, 32, 40, 40, False), (BF16, 2, 9, 16, 0, False, True, 6, 3, 12, 12, False), (BF16, 1, 5, 72, 16, False, False, 30, 1, 25, 25, False),
    (BF16, 1, 1, 8, 0, False, False, 2, 2, 1, 1, False), (BF16, 2, 40, 256, 256, False, True, 2, 8, 9, 9, False)]


def append_args(rng, case):
    dtype, L, H, D, rot, pairs, norm, blocks, page, rows, count, own = case
    n_pos = 50
    k, v = heads(rng, (L, rows, H, D), dtype), heads(rng, (L, rows, H, D), dtype)
    slot, src, pos = entries(rng, blocks * page, rows, count, n_pos)
    cs = table(rot, n_pos, rng) if rot else None
    w = (1 + 0.2 * rng.normal(size=(L, D))).astype(np.float32) if norm else None
    kw = dict(src_row=dev(src, torch.int32) if own else None, pos=dev(pos, torch.int32), cos=dev(cs[0]) if rot else None,
              sin=dev(cs[1]) if rot else None, k_weight=dev(w) if norm else None, eps=EPS, pairs=pairs)
    done = []   # (entry, slot, row, position)
    for t in range(count):
        row = int(src[t]) if own else t
        if 0 <= slot[t] < blocks * page and 0 <= row < rows and (not rot or 0 <= pos[t] < n_pos):
            done.append((int(slot[t]), row, int(pos[t])))
    turned = lambda layer, row, h, at: HO.turned(floats(k[layer, row, h]), cs[0][at] if rot else None, cs[1][at] if rot else None,
                                                 w[layer] if norm else None, EPS, pairs)
    return k, v, dev(slot, torch.int32), kw, done, turned


@pytest.mark.parametrize("case", APPEND)
@pytest.mark.parametrize("layout", ["tokens", "heads"])
def test_append(case, layout):
    dtype, L, H, D, rot, pairs, norm, blocks, page, rows, count, own = case
    rng = np.random.default_rng(D + L + count)
    k, v, slot, kw, done, turned = append_args(rng, case)
    if layout == "tokens":
        cache = [heads(rng, (L, blocks, page, H, D), dtype) for _ in range(2)]
    else:
        cache = [heads(rng, (L, blocks, H, page, D), dtype).transpose(2, 3) for _ in range(2)]
    want = [x.cpu().clone() for x in cache]
    for s, row, at in done:
        for layer in range(L):
            for h in range(H):
                want[0][layer, s // page, s % page, h] = rounded(turned(layer, row, h, at), dtype)
                want[1][layer, s // page, s % page, h] = v[layer, row, h].cpu()
    B.spec_cache_append(k, v, slot, *cache, **kw)
    assert same(cache[0], want[0]) and same(cache[1], want[1])
    if L == 1:   # the form without layers
        again = [torch.zeros_like(x[0]) for x in cache]
        first = [x.clone() for x in again]
        one = dict(kw, k_weight=None if kw["k_weight"] is None else kw["k_weight"][0])
        B.spec_cache_append(k[0], v[0], slot, *again, **one)
        B.spec_cache_append(k, v, slot, *[x.unsqueeze(0) for x in first], **kw)
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


def test_append_without_rotation_is_the_store():
    rng = np.random.default_rng(4)
    k, v = heads(rng, (2, 9, 3, 40), F32), heads(rng, (2, 9, 3, 40), F32)
    slot, src = dev([3, -1, 20, 7, 31], torch.int32), dev([8, 0, 1, 9, 5], torch.int32)
    a, b = [[torch.zeros((2, 4, 8, 3, 40), device="cuda") for _ in range(2)] for _ in range(2)]
    B.spec_cache_append(k, v, slot, *a, src_row=src)
    B.spec_cache_store(k, v, slot, *b, src_row=src)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- four bits ------------------------------------------------------------------------------------------------------

def packed_cache(L, blocks, page, H, D, layout="tokens", value=None):
    shape = (L, blocks, page, H) if layout == "tokens" else (L, blocks, H, page)
    make = lambda n: (torch.randint(0, 256, (*shape, n), dtype=torch.uint8, device="cuda") if value is None else
                      torch.full((*shape, n), value, dtype=torch.uint8, device="cuda"))
    got = [make(n) for n in (D // 2, D // 2, D // 32, D // 32)]
    return got if layout == "tokens" else [x.transpose(2, 3) for x in got]


PACK = [(BF16, 1, 4, 128, 128, False, True, 5, 16, 30, 30, False), (BF16, 3, 2, 64, 32, True, True, 4, 7, 20, 11, True),
        (BF16, 2, 3, 32, 32, False, False, 3, 5, 9, 14, True), (BF16, 1, 1, 256, 112, False, True, 2, 32, 40, 40, False),
        (BF16, 2, 9, 96, 0, False, True, 6, 3, 12, 12, False), (BF16, 1, 5, 160, 160, True, False, 30, 1, 25, 25, False),
        (BF16, 1, 1, 32, 0, False, False, 2, 2, 1, 1, False), (BF16, 2, 40, 256, 256, False, True, 2, 8, 9, 9, False), (BF16, 1, 3, 224, 48, False, True, 3, 9, 20, 20, False)]


@pytest.mark.parametrize("case", PACK)
@pytest.mark.parametrize("layout", ["tokens", "heads"])
def test_pack_and_load(case, layout):
    dtype, L, H, D, rot, pairs, norm, blocks, page, rows, count, own = case
    rng = np.random.default_rng(D + L + count)
    k, v, slot, kw, done, turned = append_args(rng, case)
    cache = packed_cache(L, blocks, page, H, D, layout)
    want = [x.cpu().clone() for x in cache]
    for s, row, at in done:
        for layer in range(L):
            for h in range(H):
                for i, x in enumerate((turned(layer, row, h, at), floats(v[layer, row, h]))):
                    scales, codes = HO.pack(x)
                    want[i][layer, s // page, s % page, h] = torch.from_numpy(HO.packed_bytes(codes))
                    want[2 + i][layer, s // page, s % page, h] = torch.from_numpy(scales)
    B.spec_packed_append(k, v, slot, *cache, **kw)
    for x, y in zip(cache, want):
        assert torch.equal(x.cpu(), y)
    # back: some slots twice, some that are none
    slots = np.concatenate([rng.integers(0, blocks * page, 20), [-1, blocks * page, 0, 0]])
    out = [torch.full((L, H, len(slots), D), -3.0, dtype=BF16, device="cuda").transpose(1, 2) for _ in range(2)]
    B.spec_packed_load(*cache, dev(slots, torch.int32), *out)
    for i in range(2):
        for t, s in enumerate(slots):
            for layer, h in np.ndindex(L, H):
                got = exact_float(out[i][layer, t, h])
                if 0 <= s < blocks * page:
                    assert np.array_equal(got, HO.values(want[2 + i][layer, s // page, s % page, h].numpy(), want[i][layer, s // page, s % page, h].numpy()), equal_nan=True)
                else:
                    assert (got == -3).all()


def test_pack_edges():
    """Zeros, the borders between codes and between scales, sizes from subnormal to the largest, infinities and NaN."""
    rows = [np.zeros(32), -np.zeros(32)]
    edges = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7]
    for e in (-133, -126, -124, -20, 0, 60, 120, 124):
        for top in (4, 5, 6, 7, 7.0625, 7.9375):
            x = np.array([top] + edges + [-y for y in edges])
            rows.append(np.resize(x * 2.0 ** e, 32))
            rows[-1][0] = top * 2.0 ** e
    for bad in (np.inf, -np.inf, np.nan):
        rows.append(np.linspace(-3, 3, 32))
        rows[-1][7] = bad
    rows.append(np.full(32, 3.38953139e38))
    rows.append(np.resize([3.38953139e38, 2.0 ** 125, -2.0 ** 124], 32))
    x = rounded(np.stack(rows).astype(np.float32), BF16)
    n = len(rows)
    new = x.cuda().view(n, 1, 32)
    cache = packed_cache(1, n, 1, 1, 32, value=0x5a)
    B.spec_packed_append(new, new, dev(np.arange(n), torch.int32), *[c[0] for c in cache])
    for i in range(n):
        scales, codes = HO.pack(floats(x[i]))
        for j in range(2):
            assert cache[2 + j][0, i, 0, 0].tolist() == scales.tolist(), rows[i]
            assert cache[j][0, i, 0, 0].tolist() == HO.packed_bytes(codes).tolist(), rows[i]


def test_load_of_every_scale_and_code():
    codes = torch.arange(256, dtype=torch.uint8)
    cache = [codes.view(16, 16).repeat(256, 1, 1).contiguous().cuda() for _ in range(2)]                       # [256 slots, 16 heads, 16 bytes]
    scale = [torch.arange(256, dtype=torch.uint8).view(256, 1, 1).expand(256, 16, 1).contiguous().cuda() for _ in range(2)]
    cache, scale = [x.unsqueeze(1) for x in cache], [x.unsqueeze(1) for x in scale]
    out = [torch.zeros((256, 16, 32), dtype=BF16, device="cuda") for _ in range(2)]
    B.spec_packed_load(*cache, *scale, dev(np.arange(256), torch.int32), *out)
    for s in range(256):
        want = np.stack([HO.values(np.array([s], np.uint8), np.arange(16 * h, 16 * h + 16).astype(np.uint8)) for h in range(16)])
        for x in out:
            assert np.array_equal(exact_float(x[s]), want, equal_nan=True), s


def test_large_caches():
    """Offsets beyond 2^32: the last block of a cache of six GiB of codes, and of one of bfloat16."""
    blocks, page, H, D = 3000, 2048, 16, 128
    rng = np.random.default_rng(2)
    codes = [torch.zeros((blocks, page, H, D // 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scale = [torch.zeros((blocks, page, H, D // 32), dtype=torch.uint8, device="cuda") for _ in range(2)]
    new = heads(rng, (3, H, D), BF16)
    last = blocks * page - 1
    slot = dev([last, 0, last - page], torch.int32)
    B.spec_packed_append(new, new, slot, *codes, *scale)
    out = [torch.zeros((3, H, D), dtype=BF16, device="cuda") for _ in range(2)]
    B.spec_packed_load(*codes, *scale, slot, *out)
    small = packed_cache(1, 3, 1, H, D, value=0)
    B.spec_packed_append(new, new, dev([0, 1, 2], torch.int32), *[x[0] for x in small])
    for i in range(2):
        assert torch.equal(codes[i].flatten(0, 1)[[last, 0, last - page]], small[i][0, :, 0])
        assert torch.equal(out[i], out[0]) and out[i].any()
    del codes, scale
    cache = [torch.zeros((blocks // 3, page, H, D), dtype=BF16, device="cuda") for _ in range(2)]
    last = blocks // 3 * page - 1
    B.spec_cache_append(new, new, dev([last, 0, last - page], torch.int32), *cache)
    assert torch.equal(cache[1].flatten(0, 1)[[last, 0, last - page]], new)


def test_append_and_load_captured():
    rng = np.random.default_rng(12)
    cs = [dev(x) for x in table(64, 100, rng)]
    new = [heads(rng, (6, 2, 64), BF16) for _ in range(2)]
    slot, pos = dev([0, 1, 2, 3, -1, 9], torch.int32), dev([4, 5, 6, 7, 0, 99], torch.int32)
    cache = [x[0] for x in packed_cache(1, 4, 4, 2, 64, value=0)]
    plain = [torch.zeros((4, 4, 2, 64), dtype=BF16, device="cuda") for _ in range(2)]
    out = [torch.zeros((6, 2, 64), dtype=BF16, device="cuda") for _ in range(2)]

    def step(cache, plain, out):
        B.spec_packed_append(*new, slot, *cache, pos=pos, cos=cs[0], sin=cs[1])
        B.spec_cache_append(*new, slot, *plain, pos=pos, cos=cs[0], sin=cs[1])
        B.spec_packed_load(*cache, slot, *out)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cache, plain, out)
    for turn in range(4):
        new[0].copy_(heads(rng, (6, 2, 64), BF16))
        pos.copy_(dev(rng.integers(0, 100, 6), torch.int32))
        slot.copy_(dev(rng.permutation(16)[:6], torch.int32))
        for x in (*cache, *plain, *out):
            x.zero_()
        want = [[x.clone() for x in y] for y in (cache, plain, out)]
        step(*want)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((*cache, *plain, *out), (*want[0], *want[1], *want[2])):
            assert torch.equal(x, y)


def test_nothing_to_do():
    z = lambda *s, t=BF16: torch.zeros(s, dtype=t, device="cuda")
    none = dev([], torch.int32)
    cache = [x[0] for x in packed_cache(1, 2, 2, 2, 32, value=7)]
    B.spec_packed_append(z(0, 2, 32), z(0, 2, 32), none, *cache)
    B.spec_packed_append(z(0, 2, 32), z(0, 2, 32), dev([1], torch.int32), *cache)
    B.spec_packed_load(*cache, none, z(0, 2, 32), z(0, 2, 32))
    assert all((x == 7).all() for x in cache)
    plain = [z(2, 2, 2, 32) for _ in range(2)]
    B.spec_cache_append(z(0, 2, 32), z(0, 2, 32), none, *plain)
    torch.cuda.synchronize()
