"""Slow CPU oracle of norms and rotation of heads and of the cache of four bits, written from their definitions: numpy, loops.

`turned` rounds as the definition says (float32, every operation by itself, the norm's mean and root in 64 bits); `turned64` is the
same in 64 bits.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

AMOUNTS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
NAN_SCALE = 255


def _pairs(rot, pairs):
    half = rot // 2
    first = np.arange(half) * (2 if pairs else 1)
    return first, first + (1 if pairs else half)


def turned(x, cos, sin, weight, eps, pairs):
    """One head [D] float32 at one position (cos, sin [half] float32, or None), in float32."""
    x = x.astype(np.float32)
    if weight is not None:
        inv = np.float32(1.0 / np.sqrt((x.astype(np.float64) ** 2).sum() / len(x) + eps))
        x = (x * inv) * weight
    if cos is not None:
        a, b = _pairs(2 * len(cos), pairs)
        y = x.copy()
        y[a] = x[a] * cos - x[b] * sin
        y[b] = x[b] * cos + x[a] * sin
        x = y
    assert x.dtype == np.float32
    return x


def turned64(x, cos, sin, weight, eps, pairs):
    """(result, sum of the sizes of what is added) of one head in 64 bits."""
    x = x.astype(np.float64)
    if weight is not None:
        x = x / np.sqrt((x ** 2).mean() + eps) * weight
    size = np.abs(x)
    if cos is not None:
        a, b = _pairs(2 * len(cos), pairs)
        y = x.copy()
        y[a] = x[a] * cos - x[b] * sin
        y[b] = x[b] * cos + x[a] * sin
        size[a] = np.abs(x[a] * cos) + np.abs(x[b] * sin)
        size[b] = np.abs(x[b] * cos) + np.abs(x[a] * sin)
        x = y
    return x, size


def pack(x):
    """(scale bytes [D / 32], codes [D]) of one head in float32."""
    scales, codes = [], []
    for g in x.astype(np.float64).reshape(-1, 32):
        if not np.isfinite(g).all():
            scales.append(NAN_SCALE)
            codes += [0] * 32
            continue
        most, e = np.abs(g).max(), -125
        while most > 7 * 2.0 ** e and e < 125:
            e += 1
        scales.append(e + 127)
        for v in g:
            off = np.abs(AMOUNTS - abs(v) / 2.0 ** e)
            near = np.flatnonzero(off == off.min())
            code = int(near[0] if len(near) == 1 else near[near % 2 == 0][0])
            codes.append(code + (8 if np.signbit(v) else 0))
    return np.array(scales, np.uint8), np.array(codes, np.uint8)


def packed_bytes(codes):
    return (codes[0::2] + 16 * codes[1::2]).astype(np.uint8)


def values(scales, packed):
    """Values [D] float64 of one head's scale bytes and bytes of codes; 2^128 and more, which no append writes, are infinite."""
    codes = np.stack([packed & 15, packed >> 4], -1).reshape(-1)
    v = AMOUNTS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == NAN_SCALE, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    v = v * np.repeat(s, 32)
    return np.where(np.abs(v) >= 2.0 ** 128, np.copysign(np.inf, v), v)
