"""fp64 oracle of the rows between a projection and the attention: norms per head and position rotation.

numpy only, written from the definitions; angles are reduced in long double, so that they hold for every 32-bit position.
"""
from __future__ import annotations

import numpy as np

TWO_PI = np.longdouble("6.283185307179586476925286766559005768")


def norm(x, weight, eps):
    """x [..., 128]: each head over the root of the mean of its squares plus eps, times weight."""
    x = np.asarray(x, np.float64)
    return x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + float(np.float32(eps))) * np.asarray(weight, np.float64)


def angles(positions, inv_freq):
    """[n, rot_dim / 2] in [0, 2 pi)."""
    full = np.asarray(positions, np.int64).astype(np.longdouble)[:, None] * np.asarray(inv_freq, np.float64).astype(np.longdouble)
    return np.mod(full, TWO_PI).astype(np.float64)


def pairs(rot_dim, interleaved):
    """(first, second) value of each pair."""
    i = np.arange(rot_dim // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot_dim // 2)


def turn(x, positions, inv_freq, interleaved, factor=1.0):
    """x [n, heads, 128] turned by the tokens' positions."""
    x = np.array(x, np.float64)
    a = angles(positions, inv_freq)
    c, s = (f(a)[:, None] * float(np.float32(factor)) for f in (np.cos, np.sin))
    first, second = pairs(2 * len(inv_freq), interleaved)
    u, w = x[..., first], x[..., second]
    x[..., first], x[..., second] = u * c - w * s, u * s + w * c
    return x


def rows(x, positions, inv_freq=None, interleaved=False, factor=1.0, weight=None, eps=1e-6):
    """What a head's values become, and how far an implementation in 32 bits with one rounding to bf16 may be off, value by value.

    The rounding: half a step, 2^-8 of the value; 2^-9 of that more where the value in 32 bits lies beyond a power of two.
    In front of it: the sum of 128 squares (16 in a row, 3 levels, each 2^-24, half of which survives the root: 10 x 2^-24), the
    root and three products (1 to 2 units each: 6 x 2^-24), cosine and sine (2.5e-8 of series, 6 roundings of at most
    2^-24: 7 x 2^-24 with the factor) and the rotation (3 x 2^-24): 26 x 2^-24 of |a| + |b|, held to 2^-19 = 32 x 2^-24."""
    y = np.asarray(x, np.float64)
    if weight is not None:
        y = norm(y, weight, eps)
    size = np.abs(y)
    if inv_freq is not None:
        first, second = pairs(2 * len(inv_freq), interleaved)
        both = (size[..., first] + size[..., second]) * max(1.0, abs(factor))
        size = size.copy()
        size[..., first] = size[..., second] = both
        y = turn(y, positions, inv_freq, interleaved, factor)
    return y, np.abs(y) * 2.0 ** -8 * (1 + 2.0 ** -9) + size * 2.0 ** -19 + 1e-38
