"""GPU parity of the attention weights of cached keys and of eviction by them.

Bounds of a weight, a sum of n probabilities p: a score's float32 sum is off by at most
(D + 4) 2^-24 scale |q| |k|, the scaled difference to the log-sum-exp (which is taken as
given) by 2 * 2^-24 of the larger of the two, the exponential by 2^-22, and the sum by
n 2^-24: each that share of p, or of the sum.  Eviction: exact, every byte of the caches."""
import numpy as np
import pytest
import torch

from oracle import kv4
from oracle.attention import paged_attention
from paper_2605_11232_amd import binding as B, synth
from tests.parity import say
from tests.test_gpu_kv4 import Cache
from tests.test_gpu_kv8 import dev, meta, rows_of, tables

pytestmark = pytest.mark.gpu
POS = np.array([(o & ~12) | ((o & 4) << 1) | ((o & 8) >> 1) for o in range(16)])


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


class WideCache:
    """A bf16 or float32 cache of random bits (finite ones)."""

    def __init__(self, nb, hkv, d, dtype, seed=0):
        g = torch.Generator("cuda").manual_seed(seed + 1)
        t = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
        self.bits = torch.int16 if dtype == "bf16" else torch.int32
        self.k = torch.randn((nb, hkv, d // 32, 16, 32), device="cuda", generator=g).to(t)
        self.v = torch.randn((nb, hkv, d, 16), device="cuda", generator=g).to(t)
        self.scales = None
        self.shape = nb, hkv, 16, d

    def raw(self):
        """Bits of keys and values as [NB, Hkv, 16, D]."""
        k = self.k.view(self.bits).cpu().numpy()[:, :, :, POS].transpose(0, 1, 3, 2, 4)
        return k.reshape(self.shape), self.v.view(self.bits).cpu().numpy().transpose(0, 1, 3, 2).copy()

    def values(self):
        k = self.k.double().cpu().numpy()[:, :, :, POS].transpose(0, 1, 3, 2, 4).reshape(self.shape)
        return k, self.v.double().cpu().numpy()


def cache_of(kind, nb, hkv, d, seed=0):
    if kind != "kv4":
        return WideCache(nb, hkv, d, kind, seed)
    c = Cache(nb, hkv, d, seed)
    c.scales.copy_(torch.randint(120, 130, c.scales.shape, device="cuda",
                                 generator=torch.Generator("cuda").manual_seed(seed)).to(torch.uint8))
    return c


# ---- weights ----------------------------------------------------------------------------------

def reference(q, kc, table, lens, cu, lse, hkv, scale):
    """Weights [n, Hkv, L] and their bounds (see the head of this file), in float64."""
    d, G = q.shape[2], q.shape[1] // hkv
    out, bound = [], []
    for r, L in enumerate(lens):
        n = int(cu[r + 1] - cu[r])
        t = np.arange(L)
        K = kc[np.asarray(table[r])[t // 16], :, t % 16, :].astype(np.float64)  # [L, Hkv, D]
        w, e = np.zeros((hkv, L)), np.zeros((hkv, L))
        for h in range(hkv):
            Q = q[cu[r]:cu[r + 1], h * G:(h + 1) * G].reshape(n * G, d)
            z = lse[cu[r]:cu[r + 1], h * G:(h + 1) * G].reshape(n * G, 1)
            ok = np.isfinite(z[:, 0])
            with np.errstate(invalid="ignore"):
                s = scale * (Q @ K[:, h].T)
                p = np.where(t[None] <= L - n + np.arange(n * G)[:, None] // G, np.exp(s - z), 0.0)
            p = np.where(ok[:, None], p, 0.0)
            ds = (d + 4) * 2.0 ** -24 * scale * np.linalg.norm(Q, axis=1)[:, None] * np.linalg.norm(K[:, h], axis=1)
            ds = ds + 2 * 2.0 ** -24 * np.maximum(np.abs(s), np.abs(z)) + 2.0 ** -22 + n * G * 2.0 ** -24
            w[h], e[h] = p.sum(0), np.where(ok[:, None], p * np.where(ok[:, None], ds, 0), 0).sum(0)
        out.append(w)
        bound.append(1.01 * e + 1e-37)
    return out, bound


# (q heads, kv heads, head_dim, query tokens, lengths): single keys and rows, lengths around
# 32, 128 and 256 keys, several row tiles, rows that end inside one, rows whose keys begin in
# the middle of a chunk, sequences without rows, odd groups
WEIGHTS = {
    "one": (8, 2, 128, [1], [1]),
    "decode": (8, 2, 128, [1] * 9, [1, 2, 15, 33, 127, 128, 129, 257, 1000]),
    "decode-64": (7, 1, 64, [1] * 5, [31, 32, 500, 513, 64]),
    "verify": (28, 4, 128, [5, 8, 2], [300, 8, 77]),
    "window": (8, 2, 128, [33, 64, 16], [700, 64, 2050]),
    "window-64": (12, 4, 64, [40, 7, 100], [555, 7, 356]),
    "prompt": (4, 2, 64, [300, 0, 1, 129], [300, 20, 260, 529]),
    "prompt-128": (6, 2, 128, [260, 515], [261, 515]),
    "wide-group": (64, 1, 128, [3, 1], [100, 290]),
    "one-head-each": (4, 4, 64, [1, 3, 90], [70, 33, 95]),
    "odd-group": (33, 1, 128, [4, 2], [40, 129]),
    # enough sequences that workgroups of many keys are chosen, lengths of one and more of them
    "sequences": (12, 4, 128, [22 + 13 * i % 79 for i in range(24)], [150 + 97 * i % 551 for i in range(24)]),
    "sequences-64": (24, 8, 64, [11 + 9 * i % 50 for i in range(36)], [64 + 31 * i % 190 for i in range(36)]),
    # and prompts, whose first workgroups go first
    "prompts": (12, 4, 128, [70 + 11 * i % 130 for i in range(80)],
                [70 + 11 * i % 130 + 20 * (i % 3) for i in range(80)]),
    "prompts-64": (24, 8, 64, [41 + 17 * i % 90 for i in range(70)], [41 + 17 * i % 90 for i in range(70)]),
    # few sequences: workgroups of 64 keys
    "some": (8, 4, 128, [90, 33, 140, 61, 100, 75], [700, 1033, 340, 61, 905, 500]),
    "some-64": (16, 8, 64, [40, 77, 120], [840, 1277, 620]),
    # prompts among requests of few rows, one behind the first 64 sequences, and sequences
    # without rows
    "mixed": (8, 2, 128, [1] * 9 + [150, 0, 1, 40, 33, 32] + [1] * 3, [300 + 57 * i for i in range(18)]),
    "mixed-64": (4, 1, 64, [1] * 70 + [200, 2, 0, 0, 17, 16, 90], [201 + 13 * i % 400 for i in range(77)]),
    "mixed-prompts": (32, 8, 128, [1] * 41 + [300, 500, 77], [500 + 31 * i % 700 for i in range(44)]),
    # one sequence, more tiles of rows than a workgroup has wavefronts
    "long-prompt": (28, 4, 128, [301], [777]),
    "long-prompt-64": (64, 8, 64, [150], [150]),
}


@pytest.mark.parametrize("cache", ["bf16", "kv4"])
@pytest.mark.parametrize("name", list(WEIGHTS))
def test_weights(name, cache):
    hq, hkv, d, q_lens, lens = WEIGHTS[name]
    say("[evict] weights", name, cache)
    r = np.random.default_rng(len(name))
    table, nb = tables(lens, 3)
    c = cache_of(cache, nb, hkv, d)
    m = meta(table, lens, q_lens)
    q = rows_of(r, sum(q_lens), hq, d, "bf16")
    kc, vc = c.values()
    _, lse = paged_attention(q, kc, vc, *m, hkv)
    lse = lse.astype(np.float32)
    if lse.size > 20:  # rows that do not count
        lse.reshape(-1)[[3, 11]] = [-np.inf, np.nan]
    width = max(lens) + 5
    n = len(lens)
    w = torch.full((n + 1, hkv, width), 7.0, device="cuda")
    args = (dev(q, torch.bfloat16), dev(lse), c.k, *map(dev, m))
    B.attention_weights(*args, w, scales=c.scales)
    first = w.clone()
    B.attention_weights(*args, w, scales=c.scales, accumulate=True)
    again = torch.empty_like(w)
    B.attention_weights(*args, again, scales=c.scales)
    torch.cuda.synchronize()
    ref, bound = reference(q.astype(np.float64), kc, table, lens, m[2], lse.astype(np.float64), hkv, d ** -0.5)
    worst = 0.0
    for i in range(n):
        got = first[i].double().cpu().numpy()
        if q_lens[i] == 0:
            assert (got == 7).all()
            continue
        err = np.abs(got[:, :lens[i]] - ref[i])
        worst = max(worst, np.max(err / bound[i]))
        assert np.all(err <= bound[i]), i
        assert (got[:, lens[i]:] == 7).all()
        assert torch.equal(again[i, :, :lens[i]], first[i, :, :lens[i]])
        # a call adds its rows to an array in at most one piece per 16 rows, each rounded to
        # 2^-24 of the sum so far, which is at most the last one: so was the first call's
        pieces = -(-q_lens[i] * (hq // hkv) // 16)
        x = first[i, :, :lens[i]].double()
        assert torch.all((w[i, :, :lens[i]].double() - 2 * x).abs() <= 4 * pieces * 2.0 ** -24 * x)
    say(f"[evict] {name}: worst {worst:.2f} of the bound")
    assert (first[n] == 7).all()
    # an array narrower than the sequences: the keys that fit.  How the rows are divided goes by
    # the array's width, too, so that a sum's order may be another; it is as near the formula.
    narrow = torch.full((n, hkv, max(1, max(lens) // 2)), 7.0, device="cuda")
    B.attention_weights(*args, narrow, scales=c.scales)
    torch.cuda.synchronize()
    for i in range(n):
        x = min(lens[i], narrow.shape[2]) if q_lens[i] else 0
        got = narrow[i].double().cpu().numpy()
        assert np.all(np.abs(got[:, :x] - ref[i][:, :x]) <= bound[i][:, :x]) and (got[:, x:] == 7).all()


@pytest.mark.parametrize("cache", ["bf16", "kv4"])
@pytest.mark.parametrize("q_lens", [[3, 2], [70, 1, 9]])
def test_weights_of_keys_that_are_not_finite(q_lens, cache):
    """An infinite key gives nothing to rows whose score is minus infinity, and rows that do
    not count (their log-sum-exp is not finite, as where such a key makes it so) give nothing to
    any key; neither do the rows that fill a tile up, nor those that do not see the key."""
    hq, hkv, d = 8, 2, 128
    lens = [x + 60 for x in q_lens]
    say("[evict] weights of keys that are not finite", q_lens, cache)
    r = np.random.default_rng(71)
    table, nb = tables(lens, 3)
    c = cache_of(cache, nb, hkv, d)
    m = meta(table, lens, q_lens)
    q = rows_of(r, sum(q_lens), hq, d, "bf16")
    q[:, :, 3] = np.where(q[:, :, 3] == 0, 1, q[:, :, 3])
    kc, _ = c.values()
    _, lse = paged_attention(q, kc, c.values()[1], *m, hkv)
    lse = lse.astype(np.float32)
    for i, L in enumerate(lens):  # the last key but one; rows that see it with a score that is not finite
        seen = slice(m[2][i + 1] - min(2, q_lens[i]), m[2][i + 1])
        lse[seen] = np.where(q[seen, :, 3] > 0, np.nan, lse[seen]) if cache == "bf16" else -np.inf
    want, got = (torch.full((len(lens), hkv, max(lens)), 7.0, device="cuda") for _ in range(2))
    args = (dev(q, torch.bfloat16), dev(lse), c.k, *map(dev, m))
    B.attention_weights(*args, want, scales=c.scales)
    for i, L in enumerate(lens):
        block, slot = int(table[i][(L - 2) // 16]), (L - 2) % 16
        if cache == "bf16":
            c.k[block, :, 0, int(POS[slot]), 3] = float("inf")
        else:
            c.scales[block, :, 0, slot] = 255
    B.attention_weights(*args, got, scales=c.scales)
    torch.cuda.synchronize()
    for i, L in enumerate(lens):
        want[i, :, L - 2] = 0
        assert torch.equal(got[i], want[i]), i


def test_weights_of_an_attention_call():
    """From the attention call's own log-sum-exps: each row's weights sum to one, and to
    the scale that the caller gives."""
    hq, hkv, d, lens = 8, 2, 128, [900, 77]
    table, nb = tables(lens, 4)
    c = cache_of("kv4", nb, hkv, d, 4)
    m = meta(table, lens, [1, 1])
    q = dev(rows_of(np.random.default_rng(4), 2, hq, d, "bf16"), torch.bfloat16)
    plan, info = B.plan(B.KIND_DECODE, 1, m[1], m[2], hq, hkv, d, 16, B.PA_BF16_KV4)
    out, lse = torch.empty_like(q), torch.empty((2, hq), device="cuda")
    ws = torch.empty(max(16, int(info.workspace_bytes)), dtype=torch.uint8, device="cuda")
    w = torch.zeros((2, hkv, 900), device="cuda")
    dm = [dev(x) for x in m]
    B.kv4_attention(B.KIND_DECODE, q, *c.args, *dm, dev(plan), info, ws, out, lse, scale=0.03)
    B.attention_weights(q, lse, c.k, *dm, w, scales=c.scales, scale=0.03)
    torch.cuda.synchronize()
    # the log-sum-exp is within 2^-16 of itself, the scores' bound is smaller
    total = w.double().sum(2)
    assert torch.all((total - hq // hkv).abs() <= hq // hkv * 2.0 ** -12)


# ---- eviction ---------------------------------------------------------------------------------

def kept_of(w, L, B_, F, W):
    """Positions that stay of weights w [L]."""
    F = min(max(F, 0), B_)
    W = min(W, B_ - F)
    x = np.where(np.isnan(w), np.inf, w)
    # NaN before infinity, then the larger, then the earlier
    order = np.lexsort((np.arange(L), -x, ~np.isnan(w)))
    order = [i for i in order if F <= i < L - W]
    return np.sort(np.concatenate([np.arange(F), order[:B_ - F - W], np.arange(L - W, L)])).astype(int)


# (lengths, new lengths, first, window): a token kept, all kept, more than all, none; lengths
# around a block; firsts inside a block, at its end, behind the new length; windows of nothing
# and larger than what stays; a sequence too long for its table's array; more positions than a
# round of the selection takes
EVICT = {
    "small": ([1, 2, 16, 17, 40], [1, 1, 5, 17, 100], [0, 0, 3, 2, 0], 0),
    "edges": ([33, 64, 48, 50, 20], [16, 17, 32, 0, -3], [16, 15, 40, 0, 0], 4),
    "windows": ([300, 257, 31], [100, 60, 30], [0, 20, 31], 64),
    "long": ([5000, 1100, 2049], [1000, 1000, 64], [100, 0, 33], 16),
    "most": ([3000, 700], [2999, 690], [1, 0], 1),
}


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("cache, d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128),
                                      ("kv4", 128), ("kv4", 64)])
@pytest.mark.parametrize("name", list(EVICT))
def test_evict(name, cache, d, in_place):
    lens, new, first, window = EVICT[name]
    say("[evict]", name, cache, d, in_place)
    hkv, n = 2, len(lens)
    r = np.random.default_rng(len(name) + d)
    keep = [max(0, min(x, L)) for x, L in zip(new, lens)]
    table, nb0 = tables(lens, 6)
    fresh, more = tables(keep, 7)
    nb = nb0 + more
    new_table = np.where(fresh >= 0, fresh + nb0, -1).astype(np.int32)
    for i in range(n):  # blocks before the first that changes are the old ones
        same = min(max(first[i], 0), keep[i]) // 16
        new_table[i, :same] = table[i, :same]
    c = cache_of(cache, nb, hkv, d, len(name))
    w = np.exp(2 * r.standard_normal((n, hkv, max(lens)))).astype(np.float32)
    w[:, 0] = np.round(w[:, 0] * 2) / 2  # many equal ones
    special = np.array([0.0, -0.0, np.inf, np.nan, 1e-42, -1.5, 3e38], np.float32)
    w[:, 1, ::3] = r.choice(special, w[:, 1, ::3].shape)
    kept = torch.full((n, hkv, max(max(keep), 1) + 2), -5, dtype=torch.int32, device="cuda")
    dw = dev(w)
    out = dw if in_place else torch.full_like(dw, 7.0)
    before = [x.copy() for x in c.raw()]
    B.kv_evict(dw, dev(table), dev(np.array(lens, np.int32)), dev(np.array(new, np.int32)), c.k, c.v,
               kept, scales=c.scales, new_table=None if in_place else dev(new_table), weights_out=out,
               first=dev(np.array(first, np.int32)), window=window)
    torch.cuda.synchronize()
    want = [x.copy() for x in before]
    to = table if in_place else new_table
    got_kept, got_w = kept.cpu().numpy(), out.cpu().numpy()
    for i in range(n):
        for h in range(hkv):
            b = keep[i]
            assert (got_kept[i, h, b:] == -5).all()
            ref = w[i, h].copy() if in_place else np.full(w.shape[2], 7.0, np.float32)
            if b > 0:
                at = kept_of(w[i, h, :lens[i]].astype(np.float64), lens[i], b, first[i], window)
                assert np.array_equal(got_kept[i, h, :b], at), (i, h)
                ref[:b] = w[i, h, at]
                new_pos = np.arange(b)
                moved = new_pos >= min(max(first[i], 0), b) // 16 * 16
                src, dst = at[moved], new_pos[moved]
                for x, y in zip(want, before):
                    x[to[i, dst // 16], h, dst % 16] = y[table[i, src // 16], h, src % 16]
            assert np.array_equal(got_w[i, h].view(np.int32), ref.view(np.int32)), (i, h)
    for x, y in zip(c.raw(), want):
        assert np.array_equal(x, y)


@pytest.mark.parametrize("cache, d", [("bf16", 128), ("f32", 64), ("kv4", 64)])
def test_evict_of_many_sequences_in_place(cache, d):
    """Enough (sequence, kv-head) pairs that each is one workgroup's: the same bytes as from
    an eviction to other blocks."""
    n, hkv = 130, 4
    r = np.random.default_rng(d)
    lens = r.integers(1, 400, n)
    new = np.maximum(1, (lens * r.random(n)).astype(int))
    first = r.integers(0, 40, n)
    table, nb0 = tables(lens, 21)
    fresh, more = tables(new, 22)
    to = np.where(fresh >= 0, fresh + nb0, -1).astype(np.int32)
    for i in range(n):
        same = min(first[i], new[i]) // 16
        to[i, :same] = table[i, :same]
    c = cache_of(cache, nb0 + more, hkv, d, 23)
    w = dev(r.random((n, hkv, 400)).astype(np.float32))
    ints = [dev(x.astype(np.int32)) for x in (lens, new, first)]
    results = []
    for in_place in (False, True):  # the first leaves the old blocks as they are
        kept = torch.full((n, hkv, 400), -1, dtype=torch.int32, device="cuda")
        ww = w.clone()
        B.kv_evict(ww, dev(table), *ints[:2], c.k, c.v, kept, scales=c.scales,
                   new_table=None if in_place else dev(to), first=ints[2], window=9)
        torch.cuda.synchronize()
        at = table if in_place else to
        raw = c.raw()
        rows = [[x[at[i, np.arange(new[i]) // 16], :, np.arange(new[i]) % 16] for i in range(n)] for x in raw]
        results.append((kept, ww, rows))
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])
    for x, y in zip(results[0][2], results[1][2]):
        assert all(np.array_equal(a, b) for a, b in zip(x, y))


def test_evict_leaves_what_does_not_fit():
    """Sequences longer than the weights or the table, or that keep more than the list or the
    new table hold, stay as they are; the others are shortened.  Blocks outside the cache are
    not written."""
    hkv, d = 2, 64
    lens = [100, 90, 60, 40]
    table, nb = tables(lens, 8)
    r = np.random.default_rng(8)
    w = r.random((4, hkv, 95)).astype(np.float32)  # the first does not fit
    c = cache_of("bf16", nb + 8, hkv, d, 8)
    before = [x.copy() for x in c.raw()]
    fresh = np.array([[nb, nb + 1]] * 4, np.int32)
    fresh[2] = [nb + 2, nb + 8]  # the second of them lies outside
    kept = torch.full((4, hkv, 30), -1, dtype=torch.int32, device="cuda")
    new = np.array([20, 31, 30, 29], np.int32)  # 31 is more than the list holds
    cut = np.ascontiguousarray(table[:, :5])
    lens_in = np.array([100, 90, 60, 81], np.int32)  # the last: more than the table holds
    B.kv_evict(dev(w), dev(cut), dev(lens_in), dev(new), c.k, c.v, kept, new_table=dev(fresh),
               weights_out=torch.empty_like(dev(w)))
    torch.cuda.synchronize()
    want = [x.copy() for x in before]
    k = kept.cpu().numpy()
    assert (k[[0, 1, 3]] == -1).all()
    for h in range(hkv):
        at = kept_of(w[2, h, :60].astype(np.float64), 60, 30, 0, 0)
        assert np.array_equal(k[2, h], at)
        for x, y in zip(want, before):
            x[nb + 2, h] = y[table[2, at[:16] // 16], h, at[:16] % 16]
    for x, y in zip(c.raw(), want):
        assert np.array_equal(x, y)


@pytest.mark.parametrize("cache", ["bf16", "kv4"])
def test_evict_past_4_gib(cache):
    """Old and new blocks whose keys and values lie past 2^32 bytes."""
    hkv, d, lens, new = 8, 128, [700, 300], [130, 299]
    per = hkv * 16 * d * 2 if cache == "bf16" else hkv * 8 * d
    far = (1 << 32) // per + 500
    table, nb = tables(lens, 9)
    fresh, more = tables(new, 10)
    r = np.random.default_rng(9)
    w = r.random((2, hkv, 700)).astype(np.float32)
    small = cache_of(cache, nb + more, hkv, d, 9)
    big = [torch.empty((far + nb + more, *x.shape[1:]), dtype=x.dtype, device="cuda")
           for x in (small.k, small.v, small.scales) if x is not None]
    for x, y in zip(big, (small.k, small.v, small.scales)):
        x[far:] = y
    if cache == "bf16":
        big.append(None)
    results = []
    for (k, v, s), shift in (((small.k, small.v, small.scales), 0), (big, far)):
        kept = torch.empty((2, hkv, 299), dtype=torch.int32, device="cuda")
        at = [np.where(x >= 0, x + y + shift, -1).astype(np.int32) for x, y in ((table, 0), (fresh, nb))]
        B.kv_evict(dev(w), dev(at[0]), dev(np.array(lens, np.int32)), dev(np.array(new, np.int32)), k, v,
                   kept, scales=s, new_table=dev(at[1]), weights_out=torch.empty_like(dev(w)), window=7)
        torch.cuda.synchronize()
        results.append([x[shift:] for x in (k, v, s) if x is not None])
    for x, y in zip(*results):
        assert torch.equal(x, y)


# ---- together ---------------------------------------------------------------------------------

class Session:
    """A pool and a cache, as a serving program runs them: contexts of a shared prefix and a
    private part, decode steps that count attention weights, an eviction, further steps."""

    def __init__(self, cache, hq=8, hkv=2, d=128, seed=0):
        self.r = np.random.default_rng(seed)
        self.cache, self.hq, self.hkv, self.d = cache, hq, hkv, d
        self.pool = B.Pool(200, 16, np.random.default_rng(seed).permutation(200).astype(np.int32))
        self.c = cache_of(cache, 200, hkv, d, seed)
        self.ids = [1, 2, 3]
        prefix = list(range(100))
        # the reference: each sequence's keys and values for each kv-head, as stored
        self.keys = {s: [np.zeros((0, d))] * hkv for s in self.ids}
        self.values = {s: [np.zeros((0, d))] * hkv for s in self.ids}
        self.weights = torch.zeros((3, hkv, 1024), device="cuda")
        k0, v0 = (rows_of(self.r, 100, hkv, d, "bf16") for _ in range(2))
        for s, extra in zip(self.ids, (300, 210, 77)):
            cached = self.pool.add(s, prefix)
            self.append([s], [100 - cached], k0[cached:], v0[cached:], [k0[:cached], v0[:cached]])
            self.pool.extend(s, [1000 * s + i for i in range(extra)])
            self.append([s], [extra], *(rows_of(self.r, extra, hkv, d, "bf16") for _ in range(2)))

    def meta(self, ids, q):
        m = self.pool.metadata(ids, q, 64)
        return [m["block_table"], m["seq_lens"], m["cu_seqlens_q"]], m["slot_mapping"]

    def store(self, k, v):
        return (kv4.round_keys(k), kv4.round_values(v)) if self.cache == "kv4" else (k, v)

    def append(self, ids, q, k, v, seen=None):
        m, slots = self.meta(ids, q)
        kd, vd = dev(k, torch.bfloat16), dev(v, torch.bfloat16)
        if self.cache == "kv4":
            B.kv4_append(kd, vd, *map(dev, m), *self.c.args)
        else:
            B.kv_append(kd, vd, dev(slots), self.c.k, self.c.v)
        for i, s in enumerate(ids):
            new = [k[m[2][i]:m[2][i + 1]], v[m[2][i]:m[2][i + 1]]]
            if seen is not None:
                new = [np.concatenate([a, b]) for a, b in zip(seen, new)]
            for store, x in zip((self.keys, self.values), self.store(*new)):
                store[s] = [np.concatenate([old, x[:, h]]) for h, old in enumerate(store[s])]

    def decode(self):
        """One token of each sequence; its output against the reference, its weights counted."""
        for s in self.ids:
            self.pool.extend(s, [7])
        n, hq, hkv, d = len(self.ids), self.hq, self.hkv, self.d
        self.append(self.ids, [1] * n, *(rows_of(self.r, n, hkv, d, "bf16") for _ in range(2)))
        q = rows_of(self.r, n, hq, d, "bf16")
        m, _ = self.meta(self.ids, [1] * n)
        plan, info = B.plan(B.KIND_DECODE, 1, m[1], m[2], hq, hkv, d, 16,
                            B.PA_BF16_KV4 if self.cache == "kv4" else B.PA_BF16, block_table=m[0])
        ws = torch.empty(max(16, int(info.workspace_bytes)), dtype=torch.uint8, device="cuda")
        dq, dm = dev(q, torch.bfloat16), [dev(x) for x in m]
        out, lse = torch.empty_like(dq), torch.empty((n, hq), device="cuda")
        if self.cache == "kv4":
            B.kv4_attention(B.KIND_DECODE, dq, *self.c.args, *dm, dev(plan), info, ws, out, lse)
        else:
            B.attention(B.KIND_DECODE, dq, self.c.k, self.c.v, *dm, dev(plan), info, ws, out, lse)
        B.attention_weights(dq, lse, self.c.k, *dm, self.weights, scales=self.c.scales, accumulate=True)
        torch.cuda.synchronize()
        G, got, total = hq // hkv, out.double().cpu().numpy(), []
        for i, s in enumerate(self.ids):
            for h in range(hkv):
                K, V = self.keys[s][h], self.values[s][h]
                assert len(K) == m[1][i]
                sc = q[i, h * G:(h + 1) * G].astype(np.float64) @ K.T * d ** -0.5
                p = np.exp(sc - sc.max(1, keepdims=True))
                p /= p.sum(1, keepdims=True)
                ref, A = p @ V, p @ np.abs(V)
                # as bounds() of test_gpu_kv8; scores' sums: |q| |k| scale (D + 4) 2^-24 < 2^-12.
                # Probabilities below 2^-126 of a row's largest, and their products with a
                # value's scale, are zero in float32 and bf16: each then takes less than 2^-126
                # |v| from the sum, or 2^-126 times a code of at most 6.
                under = len(K) * 2.0 ** -126 * max(6.0, np.abs(V).max())
                assert np.all(np.abs(got[i, h * G:(h + 1) * G] - ref)
                              <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 2.0 ** -11) * A + under)
                total.append(p.sum(0))
        return total

    def shrink(self, new, first, window, in_place):
        m, _ = self.meta(self.ids, [0] * len(self.ids))
        for s, x in zip(self.ids, new):
            self.pool.compact(s, x, first, in_place)
        after, _ = self.meta(self.ids, [0] * len(self.ids))
        kept = torch.full((len(new), self.hkv, max(new)), -1, dtype=torch.int32, device="cuda")
        B.kv_evict(self.weights, dev(m[0]), dev(m[1]), dev(np.array(new, np.int32)), self.c.k, self.c.v,
                   kept, scales=self.c.scales, new_table=None if in_place else dev(after[0]),
                   first=dev(np.full(len(new), first, np.int32)), window=window)
        torch.cuda.synchronize()
        assert after[1].tolist() == list(new)
        k = kept.cpu().numpy()
        for i, s in enumerate(self.ids):
            for store in (self.keys, self.values):
                store[s] = [store[s][h][k[i, h, :new[i]]] for h in range(self.hkv)]
            assert np.array_equal(k[i, :, :first], np.tile(np.arange(first), (self.hkv, 1)))
            last = min(window, new[i] - first)  # what is left of the window
            assert np.all(k[i, :, new[i] - last:new[i]] >= m[1][i] - last)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("cache", ["bf16", "kv4"])
def test_session(cache, in_place):
    """Decode steps, an eviction (of all but the shared prefix; the whole prompt where new
    blocks take it), decode steps on what stays, and another one."""
    s = Session(cache)
    for _ in range(3):
        s.decode()
    s.shrink([200, 160, 180], 96 if in_place else 20, 8, in_place)
    for _ in range(2):
        s.decode()
    s.shrink([120, 161, 100], 96, 5, in_place)
    # columns behind the sequences hold weights of tokens that are gone
    for i, x in enumerate([120, 161, 100]):
        s.weights[i, :, x:] = 0
    s.decode()
    # the prefix is still there for other requests, what was shortened is not
    hits = s.pool.add(9, list(range(100)))
    assert hits == 96
    for i in s.ids:
        s.pool.free(i)
    assert s.pool.add(10, list(range(100)) + [1000 + i for i in range(300)]) == 96


def test_captured_weights_and_eviction():
    """Weights counted and an eviction to other blocks in a captured graph, replayed with
    other queries and eager work between."""
    hq, hkv, d, lens, new = 8, 2, 128, [700, 333], [200, 100]
    table, nb = tables(lens, 11)
    fresh, more = tables(new, 12)
    to = np.where(fresh >= 0, fresh + nb, -1).astype(np.int32)
    c = cache_of("kv4", nb + more, hkv, d, 11)
    r = np.random.default_rng(11)
    m = [dev(x) for x in meta(table, lens, [2, 2])]
    q = torch.empty((4, hq, d), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((4, hq), 5.0, device="cuda")
    w = torch.zeros((2, hkv, 700), device="cuda")
    w_out, kept = torch.zeros_like(w), torch.zeros((2, hkv, 200), dtype=torch.int32, device="cuda")
    new_lens, dto = dev(np.array(new, np.int32)), dev(to)

    def step():
        B.attention_weights(q, lse, c.k, *m, w, scales=c.scales)
        B.kv_evict(w, m[0], m[1], new_lens, c.k, c.v, kept, scales=c.scales, new_table=dto,
                   weights_out=w_out, window=4)

    def state():
        return [x.clone() for x in (w, w_out, kept, c.k, c.v, c.scales)]

    inputs = [dev(rows_of(r, 4, hq, d, "bf16"), torch.bfloat16) for _ in range(4)]
    eager = []
    for x in inputs:
        q.copy_(x)
        step()
        torch.cuda.synchronize()
        eager.append(state())
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    for i in (2, 0, 3, 1):
        q.copy_(inputs[i])
        w.zero_(), kept.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(state(), eager[i]):
            assert torch.equal(a, b)
        q.copy_(inputs[0])
        step()
        torch.cuda.synchronize()


def test_on_another_stream():
    hq, hkv, d, lens = 8, 2, 64, [100, 65]
    table, nb = tables(lens, 13)
    results = []
    for how in range(3):
        c = cache_of("bf16", nb, hkv, d, 13)
        m = [dev(x) for x in meta(table, lens, [1, 1])]
        q = dev(rows_of(np.random.default_rng(13), 2, hq, d, "bf16"), torch.bfloat16)
        lse = torch.full((2, hq), 4.0, device="cuda")
        w = torch.zeros((2, hkv, 100), device="cuda")
        kept = torch.zeros((2, hkv, 50), dtype=torch.int32, device="cuda")
        new = dev(np.array([50, 40], np.int32))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        given = side if how == 1 else None
        with torch.cuda.stream(side if how == 2 else torch.cuda.current_stream()):
            B.attention_weights(q, lse, c.k, *m, w, stream=given)
            B.kv_evict(w, m[0], m[1], new, c.k, c.v, kept, window=3, stream=given)
        side.synchronize()
        torch.cuda.synchronize()
        results.append((w, kept, c.k, c.v))
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))
