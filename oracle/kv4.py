"""float64 oracle of the 4-bit cache (test infrastructure only).

An e2m1 number is (-1)^s times one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (codes 0 .. 7).  32 dims of a
token's key, and all dims of its value, are such numbers times 2^e, e the smallest of
-100 .. 100 with amax <= 7 * 2^e: each the nearest to x, of two equally near the one of
even code, and 6 * 2^e where x is larger.  Values that share a scale with one that is not
finite become NaN.  Tokens do not depend on each other.
"""
from __future__ import annotations

import numpy as np

NUMBERS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
EXP_MIN, EXP_MAX = -100, 100


def exponents(x):
    """Exponents of x [..., n]: one for the last axis; EXP_MAX + 1 where it has a value that
    is not finite."""
    amax = np.max(np.abs(x), axis=-1)  # of a NaN: NaN
    e = np.full(amax.shape, EXP_MIN)
    for k in range(EXP_MIN, EXP_MAX):
        e[amax > np.ldexp(7.0, k)] = k + 1
    e[~np.isfinite(amax)] = EXP_MAX + 1
    return e


def codes(x):
    """Codes 0 .. 15 of numbers x, nearest, ties to the even code."""
    a = np.minimum(np.abs(x), 6.0)
    hi = np.clip(np.searchsorted(NUMBERS, a), 1, 7)
    lo = hi - 1
    below, above = a - NUMBERS[lo], NUMBERS[hi] - a
    c = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, lo)
    return c + 8 * np.signbit(x)


def quantise(x):
    """(codes [..., n], scale bytes [...]) of x [..., n], which shares a scale."""
    x = np.asarray(x, dtype=np.float64)
    e = exponents(x)
    nan = e > EXP_MAX
    c = codes(np.where(nan[..., None], 0.0, np.ldexp(x, -np.where(nan, 0, e)[..., None])))
    return np.where(nan[..., None], 0, c).astype(np.uint8), np.where(nan, 255, e + 127).astype(np.uint8)


def values(c, scale):
    """What codes [..., n] under scale bytes [...] stand for."""
    v = NUMBERS[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, np.ldexp(1.0, scale.astype(np.int64) - 127))
    return v * s[..., None]


def round_keys(k):
    """Keys [T, H, D] as the cache holds them."""
    k = np.asarray(k, dtype=np.float64)
    return values(*quantise(k.reshape(*k.shape[:-1], -1, 32))).reshape(k.shape)


def round_values(v):
    """Values [T, H, D] as the cache holds them."""
    return values(*quantise(v))
