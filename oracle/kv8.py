"""float64 oracle of the 8-bit cache (test infrastructure only).

An e4m3 number is (-1)^s * m * 2^(x - 3) with a four-bit significand: m of
8 .. 15 for x of -6 .. 8 (448 = 14 * 2^5 is the largest that is used), and
m * 2^-9, m of 0 .. 7, below.  A (block, kv-head) of keys, and of values, is
such numbers times 2^e.  Storing tokens: e is the smallest of -100 .. 120 with
amax <= 448 * 2^e over the new tokens' finite values; where the block holds
earlier tokens, no less than its e, and those are rounded again to the new one.
Rounding is to nearest, ties to even m; what is not finite becomes NaN, and finite
magnitudes above 240 * 2^120 (the number below 2^128) become that.

The store holds the values (code * 2^e) in the layout of oracle.attention
(K [NB, Hkv, bs, D], V [NB, Hkv, D, bs]) and the exponents [NB, Hkv, 2].
"""
from __future__ import annotations

import numpy as np

EXP_MIN, EXP_MAX = -100, 120
MOST = 240 * 2.0 ** 120


def round_e4m3(x):
    """Nearest e4m3 numbers of |x| <= 448 (NaN stays NaN), in float64."""
    x = np.asarray(x, dtype=np.float64)
    _, p = np.frexp(np.abs(x))                 # |x| in [2^(p-1), 2^p)
    step = np.ldexp(1.0, np.maximum(p - 1, -6) - 3)
    return np.rint(x / step) * step            # rint: ties to even


def exponent(amax: float) -> int:
    """Smallest e of EXP_MIN .. EXP_MAX with amax <= 448 * 2^e."""
    e = EXP_MIN
    while e < EXP_MAX and amax > np.ldexp(448.0, e):
        e += 1
    return e


def new_exponents(num_blocks: int, num_kv_heads: int):
    return np.zeros((num_blocks, num_kv_heads, 2), dtype=np.int64)


def _store(values, exps, off, x):
    """values [Hkv, bs, D] view of one block's keys or values, exps [Hkv]: the
    tokens x [n, Hkv, D] go to offsets off .. off + n - 1."""
    for h in range(values.shape[0]):
        rows = np.asarray(x[:, h, :], dtype=np.float64)
        fin = np.abs(rows[np.isfinite(rows)])
        e = exponent(fin.max() if fin.size else 0.0)
        if off > 0:
            old = exps[h]
            e = max(e, int(old))
            if e > old:
                values[h, :off] = np.ldexp(round_e4m3(np.ldexp(
                    values[h, :off].astype(np.float64), -e)), e)
        rows = np.where(np.isfinite(rows), np.clip(rows, -MOST, MOST), np.nan)
        values[h, off:off + len(rows)] = np.ldexp(round_e4m3(np.ldexp(rows, -e)), e)
        exps[h] = e


def append(k_cache, v_cache, exps, block_table, seq_lens, cu_seqlens, k_new, v_new):
    """Store rows cu[r] .. cu[r+1] as sequence r's last positions."""
    bs = k_cache.shape[2]
    for r in range(len(seq_lens)):
        a, b = int(cu_seqlens[r]), int(cu_seqlens[r + 1])
        pos = int(seq_lens[r]) - (b - a)
        while a < b:
            j, off = divmod(pos, bs)
            n = min(bs - off, b - a)
            blk = int(block_table[r][j])
            _store(k_cache[blk], exps[blk, :, 0], off, k_new[a:a + n])
            _store(v_cache[blk].transpose(0, 2, 1), exps[blk, :, 1], off, v_new[a:a + n])
            a += n
            pos += n


def norm_rope(x, positions, cos_sin, weight=None, eps=1e-6, norm=True, interleaved=False):
    """Heads x [T, H, D] normalised (root mean square, weight) and rotated by the
    table's angles (cosines, then sines): pairs are dims (i, i + rot / 2), or
    (2 i, 2 i + 1)."""
    x = np.asarray(x, dtype=np.float64)
    if norm:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
        if weight is not None:
            x = x * np.asarray(weight, dtype=np.float64)
    y = x.copy()
    rot = cos_sin.shape[1]
    half = rot // 2
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c = np.asarray(cos_sin, dtype=np.float64)[positions, i][:, None]
        s = np.asarray(cos_sin, dtype=np.float64)[positions, half + i][:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y
