"""The oracle of heads and of the cache of four bits against what their formulas imply (no GPU needed)."""
import numpy as np
import pytest

from oracle import heads_oracle as HO


@pytest.mark.parametrize("pairs", [False, True])
def test_rotation_keeps_pairs_sizes_and_adds_angles(pairs):
    rng = np.random.default_rng(3)
    x, a, b = rng.normal(size=24).astype(np.float32), rng.normal(size=8), rng.normal(size=8)
    turn = lambda v, t: HO.turned64(v, np.cos(t), np.sin(t), None, 0, pairs)[0]
    y = turn(x, a)
    i, j = HO._pairs(16, pairs)
    assert np.allclose(y[i] ** 2 + y[j] ** 2, x[i].astype(float) ** 2 + x[j].astype(float) ** 2, rtol=1e-12)
    assert np.array_equal(y[16:], x[16:])
    assert np.allclose(turn(y, b), turn(x, a + b), atol=1e-12)
    # the product of a query and a key hangs on the difference of their positions only
    k = rng.normal(size=24)
    assert np.isclose(turn(x, 5 * a) @ turn(k, 3 * a), turn(x, 9 * a) @ turn(k, 7 * a), rtol=1e-12)


def test_norm():
    x = np.random.default_rng(4).normal(size=64).astype(np.float32) * 7
    y = HO.turned64(x, None, None, np.full(64, 2.0), 0.0, False)[0]
    assert np.isclose((y ** 2).mean(), 4)
    assert np.allclose(HO.turned(x, None, None, np.full(64, 2, np.float32), 0.0, False), y, rtol=3 * 2.0 ** -23)


def test_packing_is_nearest_and_values_come_back():
    rng = np.random.default_rng(5)
    for size in (1e-30, 1e-3, 1.0, 6.9, 7.0, 7.1, 8.0, 1e30):
        x = (rng.normal(size=64) * size).astype(np.float32)
        x[3] = size
        s, c = HO.pack(x)
        v = HO.values(s, HO.packed_bytes(c))
        scale = np.repeat(2.0 ** (s.astype(float) - 127), 32)
        step = np.where(np.abs(x) < 2 * scale, 0.5, np.where(np.abs(x) < 4 * scale, 1, 2)) * scale
        assert (np.abs(v - x) <= step / 2).all()
        again = HO.pack(v.astype(np.float32))
        assert np.array_equal(HO.values(again[0], HO.packed_bytes(again[1])), v)
    zero = HO.pack(np.zeros(32, np.float32))
    assert zero[0][0] == 2 and not zero[1].any()
    x = np.zeros(64, np.float32)
    x[40] = np.inf
    s, c = HO.pack(x)
    assert list(s) == [2, 255] and np.isnan(HO.values(s, HO.packed_bytes(c))[32:]).all()
