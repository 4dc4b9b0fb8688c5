"""GPU parity of the 8-bit cache (append, read back, attention) and of the norms
and rotation before it, against the float64 oracle, at the sizes, masks and
values where they can go wrong.

Bounds.  Append and read back: exact, codes and scales bit for bit.  Attention
over the cache's values: the output is rounded to bf16 (2^-8 of it) and so is
each probability of the value product (2^-8 of sum_t p_t |v_t|); the scores'
float32 sums are off by at most (D + 4) 2^-24 scale |q| |k| each, which moves
probabilities by that share and the log-sum-exp by that much; exponentials,
sums and merges of float32 add less than 2^-16.  Norms and rotation: the sum of
squares (D + 4) 2^-24, seven products and sums of 2^-24 each, the output's own
rounding."""
import numpy as np
import pytest
import torch

from oracle import kv8
from oracle.attention import paged_attention
from oracle.run import OracleReplay
from paper_2605_11232_amd import binding as B, synth
from tests.parity import say
from tests.test_gpu_paths import launch_workload

pytestmark = pytest.mark.gpu
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# ---- the cache on the device as the oracle's arrays -------------------------------------------

class Cache:
    """A device cache whose every byte starts as garbage: codes at random (NaN
    codes among them), scale bytes at random."""

    def __init__(self, nb, hkv, d, seed=0):
        r = np.random.default_rng([seed, 9])
        self.nb, self.hkv, self.d = nb, hkv, d
        t = [torch.from_numpy(r.integers(0, 256, s, dtype=np.uint8)).cuda()
             for s in B.kv8_cache_shapes(nb, hkv, d)]
        self.k, self.v = t[0].view(torch.float8_e4m3fn), t[1].view(torch.float8_e4m3fn)
        self.scales = t[2]
        self.args = self.k, self.v, self.scales

    def raw(self):
        """Codes of keys and values as [NB, Hkv, 16, D], and scale bytes."""
        k = self.k.view(torch.uint8).cpu().numpy().transpose(0, 1, 3, 2, 4)
        v = self.v.view(torch.uint8).cpu().numpy().transpose(0, 1, 3, 2)
        return (k.reshape(self.nb, self.hkv, 16, self.d), v.copy(), self.scales.cpu().numpy())

    @staticmethod
    def values(codes, scale):
        t = torch.from_numpy(np.ascontiguousarray(codes)).view(torch.float8_e4m3fn).double().numpy()
        return np.ldexp(t, scale.astype(np.int64)[:, :, None, None] - 127)


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def meta(table, lens, q):
    cu = np.concatenate([[0], np.cumsum(q)]).astype(np.int32)
    return [np.asarray(table, np.int32), np.asarray(lens, np.int32), cu]


def tables(lens, seed, spare=3):
    """Disjoint random block tables, padded with -1; (table, num_blocks)."""
    n = [-(-x // 16) for x in lens]
    nb = sum(n) + spare
    ids = np.random.default_rng([seed, 1]).permutation(nb).astype(np.int32)
    out = np.full((len(lens), max(max(n, default=1), 1) + 1), -1, np.int32)
    at = 0
    for r, x in enumerate(n):
        out[r, :x] = ids[at:at + x]
        at += x
    return out, nb


def rows_of(r, T, hkv, d, dtype):
    x = r.standard_normal((T, hkv, d)) * np.exp(r.standard_normal((T, 1, 1)))
    return synth.round_to_dtype(x.astype(np.float32), dtype)


def strided(x, dtype, side):
    """x [T, H, D] as a column slice of a wider matrix of garbage."""
    T, h, d = x.shape
    wide = torch.full((T, 3 * h, d), float("nan"), dtype=dtype, device="cuda")
    wide[:, side * h:(side + 1) * h] = dev(x, dtype)
    return wide[:, side * h:(side + 1) * h]


# lengths and new tokens of a sequence of appends: one token each, inside a
# block, at its ends, over several blocks; sequences without new tokens or empty
# ones between; one token to a long context; more sequences than one round of
# the sequence search compares
APPENDS = {
    "one": (2, 128, [([1], [1])]),
    "decode": (2, 64, [([14, 15, 16, 30, 0], [14, 15, 16, 30, 0]), ([15, 16, 17, 31, 1], [1] * 5), ([16, 17, 18, 32, 2], [1] * 5),
                       ([17, 18, 19, 33, 3], [1] * 5)]),
    "ragged": (1, 128, [([0, 0, 2, 16, 16], [0, 0, 2, 16, 16]),
                        ([40, 0, 7, 16, 33], [40, 0, 5, 0, 17]), ([41, 0, 30, 48, 33], [1, 0, 23, 32, 0])]),
    "ends": (3, 64, [([0, 15, 1], [0, 15, 1]), ([16, 32, 15], [16, 17, 14]), ([17, 48, 16], [1, 16, 1])]),
    "long": (2, 128, [([1000], [1000]), ([1005], [5]), ([1029], [24])]),
    "many": (1, 64, [([1 + i % 37 for i in range(300)], [1 + i % 37 for i in range(300)]),
                     ([2 + i % 37 for i in range(300)], [1] * 300)]),
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(APPENDS))
def test_append_and_read(name, dtype):
    """Codes, scales and untouched bytes after every append, and the rows read back."""
    say("[kv8] append", name, dtype)
    hkv, d, steps = APPENDS[name]
    r = np.random.default_rng(len(name))
    table, nb = tables(steps[-1][0], 5)
    c = Cache(nb, hkv, d)
    kc, vc = np.zeros((nb, hkv, 16, d)), np.zeros((nb, hkv, d, 16))
    ex = kv8.new_exponents(nb, hkv)
    written = np.zeros((nb, 16), bool)
    rk, rv, rs = c.raw()
    for i, (lens, q) in enumerate(steps):
        T = sum(q)
        k, v = rows_of(r, T, hkv, d, dtype), rows_of(r, T, hkv, d, dtype)
        m = meta(table, lens, q)
        kv8.append(kc, vc, ex, *m, k, v)
        for n, L, row in zip(q, lens, table):
            for p in range(L - n, L):
                written[row[p // 16], p % 16] = True
        B.kv8_append(strided(k, DTYPE[dtype], 0), strided(v, DTYPE[dtype], 2), *map(dev, m), *c.args)
        torch.cuda.synchronize()
        nk, nv, ns = c.raw()
        used = written.any(1)
        assert np.array_equal(ns[used].astype(int) - 127, ex[used])
        assert np.array_equal(ns[~used], rs[~used])
        for new, before, side, ref in ((nk, rk, 0, kc), (nv, rv, 1, vc.transpose(0, 1, 3, 2))):
            hidden = ~np.broadcast_to(written[:, None, :, None], new.shape)
            assert np.array_equal(new[hidden], before[hidden]), "bytes of unused slots"
            got = c.values(new, ns[:, :, side])
            assert np.array_equal(got[~hidden], ref[~hidden])
        # read back: this step's rows, then whole contexts, packed and strided
        for n in (q, lens):
            rows = sum(n)
            mm = meta(table, lens, n)
            ko = torch.full((rows + 2, hkv, d), 7.0, dtype=DTYPE[dtype], device="cuda")
            wide = torch.full((rows, 2 * hkv, d), 7.0, dtype=DTYPE[dtype], device="cuda")
            B.kv8_read(ko[:rows], wide[:, hkv:], *map(dev, mm), *c.args)
            torch.cuda.synchronize()
            seq = np.repeat(np.arange(len(n)), n)
            pos = np.concatenate([np.arange(L - x, L) for L, x in zip(lens, n)] or [[]]).astype(int)
            blk = table[seq, pos // 16]
            assert np.array_equal(ko[:rows].double().cpu().numpy(), kc[blk, :, pos % 16])
            assert np.array_equal(wide[:, hkv:].double().cpu().numpy(), vc[blk, :, :, pos % 16])
            assert (ko[rows:] == 7).all() and (wide[:, :hkv] == 7).all()


@pytest.mark.parametrize("d", [64, 128])
def test_append_of_values_at_the_ends_of_the_range(d):
    """Zeros, the smallest and largest magnitudes, ties, scales that jump far,
    infinities and NaN (stored as NaN, kept out of the scale)."""
    hkv, r = 2, np.random.default_rng(d)
    blocks = [np.zeros(3), np.full(3, 2.0 ** -126), np.array([1e-40, 0, -1e-40]),
              np.array([3.3e38, -3.3e38, 1.0]), np.array([448.0, 448.0, -448.0]),
              np.array([449.0, 1.0, 0.0]), np.array([np.inf, 1.0, -np.inf]),
              np.array([np.nan, np.nan, np.nan]), np.array([1e-30, 1e30, 1e-30]),
              np.array([1e30, 1e-30, 1.0]), np.array([17.0, 19.0, 21.0])]
    n = len(blocks)
    x = np.stack([b[:, None, None] * np.ones((1, hkv, d)) for b in blocks])  # [n, 3, hkv, d]
    x[:, :, 1] *= r.choice([1.0, -0.5, 0.25, 2.0 ** -9], (n, 3, d))
    x = x.astype(np.float32)
    table, nb = tables([3] * n, 6)
    c = Cache(nb, hkv, d, 1)
    kc, vc = np.zeros((nb, hkv, 16, d)), np.zeros((nb, hkv, d, 16))
    ex = kv8.new_exponents(nb, hkv)
    for i in range(3):  # a token at a time
        m = meta(table, [i + 1] * n, [1] * n)
        kv8.append(kc, vc, ex, *m, x[:, i], -x[:, i])
        B.kv8_append(dev(x[:, i]), dev(-x[:, i]), *map(dev, m), *c.args)
    torch.cuda.synchronize()
    k, v, s = c.raw()
    used = table[:, 0]
    assert np.array_equal(s[used].astype(int) - 127, ex[used])
    np.testing.assert_array_equal(c.values(k, s[:, :, 0])[used, :, :3], kc[used, :, :3])
    np.testing.assert_array_equal(c.values(v, s[:, :, 1])[used, :, :3],
                                  vc.transpose(0, 1, 3, 2)[used, :, :3])
    assert np.isnan(kc[table[7, 0], 0, :3]).all() and np.isfinite(kc[table[4, 0]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_largest_finite_values_stay_finite(dtype):
    """Values whose nearest code would stand for 2^128 are stored as the largest below
    it, 240 * 2^120: read back finite, and a value of no weight adds nothing."""
    hkv, hq, d, L = 2, 4, 128, 20
    largest = float(torch.finfo(DTYPE[dtype]).max)
    table, nb = tables([L], 13)
    c = Cache(nb, hkv, d, 13)
    kc, vc = np.zeros((nb, hkv, 16, d)), np.zeros((nb, hkv, d, 16))
    ex = kv8.new_exponents(nb, hkv)
    k, v = np.zeros((L, hkv, d), np.float32), np.ones((L, hkv, d), np.float32)
    v[3, :, 0], v[3, :, 1], v[3, :, 2], v[3, :, 3] = largest, -largest, 244 * 2.0 ** 120, 236 * 2.0 ** 120
    v[17, 0], k[9, 1, 5] = 248 * 2.0 ** 120, -largest
    k[18, :, 0] = 448.0
    m = meta(table, [L], [L])
    kv8.append(kc, vc, ex, *m, k, v)
    B.kv8_append(dev(k, DTYPE[dtype]), dev(v, DTYPE[dtype]), *map(dev, m), *c.args)
    ko, vo = (torch.empty((L, hkv, d), dtype=DTYPE[dtype], device="cuda") for _ in range(2))
    B.kv8_read(ko, vo, *map(dev, m), *c.args)
    q = torch.zeros((1, hq, d), dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 16.0
    mq = meta(table, [L], [1])
    plan, info = B.plan(B.KIND_DECODE, 1, mq[1], mq[2], hq, hkv, d, 16, B.PA_BF16_KV8)
    out = torch.empty_like(q)
    B.kv8_attention(B.KIND_DECODE, q, *c.args, *map(dev, mq), dev(plan), info, None, out)
    torch.cuda.synchronize()
    seq, pos = table[0, np.arange(L) // 16], np.arange(L) % 16
    assert np.array_equal(ko.double().cpu().numpy(), kc[seq, :, pos])
    assert np.array_equal(vo.double().cpu().numpy(), vc[seq, :, :, pos])
    most = 240 * 2.0 ** 120
    assert vc[seq[3], 0, :4, 3].tolist() == [most, -most, most, 240 * 2.0 ** 120]
    assert np.abs(vc[np.isfinite(vc)]).max() == most and np.isfinite(vc).all()
    # all weight is on key 18: ones, but for kv-head 0, where they are below its block's steps
    assert np.array_equal(out.double().cpu().numpy()[0],
                          np.repeat([np.zeros(d), np.ones(d)], hq // hkv, 0))


def test_append_skips_what_it_cannot_place():
    """Block ids outside the cache, positions past the table and rows past the
    caller's write nothing; the other sequences are stored."""
    hkv, d = 2, 128
    lens, q = [20, 40, 18], [20, 4, 2]
    table, nb = tables(lens, 7)
    c, want = Cache(nb, hkv, d, 2), Cache(nb, hkv, d, 2)
    r = np.random.default_rng(3)
    k, v = rows_of(r, sum(q), hkv, d, "bf16"), rows_of(r, sum(q), hkv, d, "bf16")
    k, v = dev(k, torch.bfloat16), dev(v, torch.bfloat16)
    m = meta(table, lens, q)
    B.kv8_append(k[20:24], v[20:24], *map(dev, meta(table[1:2], [40], [4])), *want.args)
    bad = m[0].copy()
    bad[0, 0], bad[0, 1], bad[2, 1] = -1, nb, -7
    B.kv8_append(k, v, dev(bad), dev(m[1]), dev(m[2]), *c.args)
    torch.cuda.synchronize()
    assert all(np.array_equal(a, b) for a, b in zip(c.raw(), want.raw()))
    # a table of two columns: the second sequence's last tokens are past it; a row
    # count of 22: the third sequence's rows are past it; more rows than positions
    c, want = Cache(nb, hkv, d, 2), Cache(nb, hkv, d, 2)
    B.kv8_append(k[:20], v[:20], *map(dev, meta(table[:1], [20], [20])), *want.args)
    two = np.ascontiguousarray(m[0][:, :2])
    B.kv8_append(k[:22], v[:22], dev(two), dev(m[1]), dev(m[2]), *c.args)
    B.kv8_append(k, v, dev(m[0]), dev(np.array([3, 3, 1], np.int32)), dev(m[2]), *c.args)
    torch.cuda.synchronize()
    a, b = c.raw(), want.raw()
    # the last call's second sequence holds 3 positions and has 4 rows: skipped too
    assert all(np.array_equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("lens, q, n", [([20, 40, 18], [20, 4, 2], 22), ([3, 21, 9], [1, 2, 1], 2),
                                        ([40], [40], 21)])
def test_rows_past_the_callers_are_skipped(lens, q, n):
    """cu_seqlens that run past n_tokens, in the middle of a block: the rows before are
    stored, and read back, those behind are not touched."""
    hkv, d = 2, 64
    table, nb = tables(lens, 15)
    c, want = Cache(nb, hkv, d, 15), Cache(nb, hkv, d, 15)
    r = np.random.default_rng(15)
    k, v = (dev(rows_of(r, sum(q), hkv, d, "bf16"), torch.bfloat16) for _ in range(2))
    m = meta(table, lens, q)
    at = np.minimum(m[2], n)
    cut = [table, np.array(lens, np.int32) - np.diff(m[2] - at).astype(np.int32), at]
    for x in (c, want):  # what lies before the new tokens
        before = np.array(lens) - np.array(q)
        old = dev(rows_of(np.random.default_rng(16), int(before.sum()), hkv, d, "bf16"), torch.bfloat16)
        B.kv8_append(old, old, *map(dev, meta(table, before, before)), *x.args)
    B.kv8_append(k[:n], v[:n], *map(dev, cut), *want.args)
    B.kv8_append(k[:n], v[:n], *map(dev, m), *c.args)
    torch.cuda.synchronize()
    assert all(np.array_equal(a, b) for a, b in zip(c.raw(), want.raw()))
    out = torch.full((4, n + 3, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
    B.kv8_read(out[0, :n], out[1, :n], *map(dev, cut), *c.args)
    B.kv8_read(out[2, :n], out[3, :n], *map(dev, m), *c.args)
    torch.cuda.synchronize()
    assert torch.equal(out[:2], out[2:]) and (out[:, n:] == 7).all() and (out[:, :n] != 7).any()


# ---- attention --------------------------------------------------------------------------------

def bounds(q, kc, vc, table, lens, cu, hkv, out, lse):
    """Elementwise bounds of out and lse (see the head of this file)."""
    T, hq, d = q.shape
    A, _ = paged_attention(q, kc, np.abs(vc), table, lens, cu, hkv)
    ds = np.zeros((T, hq))
    for r in range(len(lens)):
        a, b = int(cu[r]), int(cu[r + 1])
        t = np.arange(int(lens[r]))
        kn = np.linalg.norm(kc[np.asarray(table[r])[t // 16], :, t % 16, :].astype(np.float64), axis=2)
        top = kn.max(0) if len(t) else np.zeros(hkv)
        ds[a:b] = np.linalg.norm(q[a:b], axis=2) * np.repeat(top, hq // hkv)[None]
    ds *= (d + 4) * 2.0 ** -24 / np.sqrt(d)
    tiny = 2.0 ** -16
    return (2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 2 * ds[..., None] + tiny) * A,
            ds + tiny * np.maximum(1, np.abs(lse)))


def check(p, q, orc, ro, hkv, label):
    md = ro["meta"]
    out, lse = p.out.double().cpu().numpy(), p.lse.double().cpu().numpy()
    bo, bl = bounds(q, orc.k_cache, orc.v_cache, md["block_table"], md["seq_lens"],
                    md["cu_seqlens_q"], hkv, ro["out"], ro["lse"])
    eo, el = np.abs(out - ro["out"]), np.abs(lse - ro["lse"])
    say(f"[kv8] {label}: worst out {np.max(eo / bo):.2f}, lse {np.max(el / bl):.2f} of the bound")
    assert np.all(eo <= bo) and np.all(el <= bl), label


def replay(cfg, q_lens, lens, seed, prefix=0, cascade=True, num_cus=0):
    from paper_2605_11232_amd.runtime import DeviceReplay
    wl = launch_workload(cfg, q_lens, lens, seed, prefix)
    dv = DeviceReplay(wl, kv8=True, cascade=cascade, num_cus=num_cus)
    # unwritten slots: NaN codes under the largest scales
    dv.k_cache.view(torch.uint8).fill_(0x7F)
    dv.v_cache.view(torch.uint8).fill_(0xFF)
    dv.scales.fill_(255)
    return wl, dv.setup(), OracleReplay(wl, kv8=True).setup()


# (q heads, kv heads, head_dim, query tokens, lengths, prefix): row items of one and
# two column tiles, part steps of 64 keys, blocks that end inside one, a single key;
# tiles whole, split, of few rows, with empty sequences between; shared prefixes;
# groups of one, of an odd number and of a whole tile; one kv-head
ATTN = {
    "one-token": (8, 2, 128, [1], [1], 0),
    "row-lengths": (8, 2, 128, [1] * 12, [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 129], 0),
    "row-lengths-64": (4, 4, 64, [1] * 8, [1, 16, 48, 64, 66, 95, 160, 1025], 0),
    "row-split": (32, 8, 128, [1] * 2, [1000, 257], 0),
    "row-long": (16, 2, 64, [1], [9001], 0),
    "row-wide": (6, 2, 64, [8] * 3, [1040, 9, 1033], 0),
    "row-wide-128": (28, 4, 128, [4] * 3, [17, 4, 700], 0),
    "rows-of-16": (16, 1, 128, [1, 2], [300, 41], 0),
    "shared": (8, 2, 128, [1] * 3, [2100, 2049, 2563], 2048),
    "shared-64": (7, 1, 64, [1] * 40, [1600 + 9 * i for i in range(40)], 1584),
    "verify-tiles": (16, 2, 128, [5] * 3, [1000, 515, 2053], 0),
    "verify-shared": (16, 2, 64, [5] * 3, [2000, 1030, 1800], 1024),
    "tile-one-step": (8, 2, 128, [40], [40], 0),
    "tile-steps": (8, 2, 128, [70, 64, 65, 17], [70, 128, 129, 257], 0),
    "tile-steps-64": (4, 1, 64, [70, 64, 65, 17], [70, 128, 129, 257], 0),
    "tile-mixed": (28, 4, 128, [65, 0, 1, 40, 1, 0], [641, 5, 1, 900, 330, 12], 0),
    "tile-split": (8, 2, 128, [100], [2100], 0),
    "tile-split-64": (4, 4, 64, [129, 3], [1300, 700], 0),
    "tile-group-128": (128, 1, 64, [3, 1], [90, 300], 0),
    "prefill-prefix": (32, 8, 128, [90, 33, 200], [602, 545, 712], 512),
    "tail": (8, 2, 64, [700] * 5, [700, 733, 764, 900, 1000], 0),
}


@pytest.mark.parametrize("name", list(ATTN))
def test_attention(name):
    attention_case(name)


@pytest.mark.parametrize("name", ["shared", "shared-64", "verify-shared"])
def test_attention_on_a_split_off_prefix(name):
    """The same launches planned for a chip so small that the shared keys are worth
    tiles of their own."""
    assert attention_case(name, num_cus=8).n_shared_items > 0


def attention_case(name, num_cus=0):
    hq, hkv, d, q_lens, lens, prefix = ATTN[name]
    say("[kv8] attention", name)
    cfg = synth.AttnConfig(f"kv8-{name}", "bf16", hq, hkv, d, 16, 7000 + len(name))
    wl, dv, orc = replay(cfg, q_lens, lens, 50, prefix, num_cus=num_cus)
    ro = orc.launch(wl.launches[0])
    p = dv.run(wl.launches[0])
    torch.cuda.synchronize()
    assert p.info.dtype == B.PA_BF16_KV8
    check(p, wl.launches[0].q.get().astype(np.float64), orc, ro, hkv, name)
    first = p.out.clone(), p.lse.clone()
    p.out.fill_(3.0), p.lse.fill_(3.0)
    dv.attend(p)  # the plan's counters are as they were
    torch.cuda.synchronize()
    assert torch.equal(p.out, first[0]) and torch.equal(p.lse, first[1])
    if p.kind == "decode" and p.info.workspace_bytes <= B.NOALLOC_WORKSPACE_BYTES:
        out, lse = torch.empty_like(p.out), torch.empty_like(p.lse)
        B.kv8_attention_decode_noalloc(p.q, dv.k_cache, dv.v_cache, dv.scales, p.block_table,
                                       p.seq_lens, p.cu, p.plan, p.info, out, lse)
        torch.cuda.synchronize()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    return p.info


def test_attention_with_tail_lists():
    """A launch with more tiles than the chip holds at once: wildcard workgroups
    take the last ones."""
    cfg = synth.AttnConfig("kv8-tail-lists", "bf16", 16, 8, 64, 16, 7100)
    wl, dv, orc = replay(cfg, [520] * 12, [520] * 12, 51)
    p = dv.run(wl.launches[0])
    torch.cuda.synchronize()
    assert p.info.variant & 4
    rows = [(t, h) for t in range(0, 520 * 12, 97) for h in (0, 7, 15)]
    ro = orc.launch(wl.launches[0], rows=rows)
    t, h = np.array(rows).T
    err = np.abs(p.out.double().cpu().numpy()[t, h] - ro["out"][t, h])
    # |o| <= sum p |v|: twice 2^-8 of the largest value and what the head of this file lists
    assert np.all(err <= (2 * 2.0 ** -8 + 2.0 ** -10) * np.abs(orc.v_cache).max())
    assert np.all(np.isfinite(p.out.float().cpu().numpy()))
    # every row against the bf16 path over the same values
    ref = bf16_attention(dv, p)
    assert torch.allclose(p.out.float(), ref.float(), rtol=2.0 ** -7, atol=2.0 ** -7)


def bf16_attention(dv, p):
    """The bf16 call over a bf16 cache of the values that the 8-bit cache holds."""
    nb, hkv, d, bs = dv.v_cache.shape
    s = torch.exp2(dv.scales.double() - 127)
    k = dv.k_cache.double() * s[:, :, 0, None, None, None]      # [nb, hkv, d / 64, 16, 64]
    k = k.view(nb, hkv, d // 64, bs, 2, 32).transpose(3, 4).reshape(nb, hkv, d // 32, bs, 32)
    off = torch.arange(bs, device="cuda")
    pos = (off & ~12) | ((off & 4) << 1) | ((off & 8) >> 1)
    kc = torch.empty((nb, hkv, d // 32, bs, 32), dtype=torch.bfloat16, device="cuda")
    kc[:, :, :, pos] = k.to(torch.bfloat16)
    vc = (dv.v_cache.double() * s[:, :, 1, None, None]).to(torch.bfloat16)
    plan, info = B.plan(p.info.kind, p.info.n_q, p.meta["seq_lens"], p.meta["cu_seqlens_q"],
                        p.info.num_q_heads, hkv, d, bs, B.PA_BF16,
                        block_table=p.meta["block_table"])
    ws = torch.empty(max(1, int(info.workspace_bytes)), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(p.out)
    B.attention(p.info.kind, p.q, kc, vc, p.block_table, p.seq_lens, p.cu, dev(plan), info, ws, out)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("scale", [1e-3, 1.0, 3.0])
def test_attention_scale(scale):
    """The caller's softmax scale, from nearly uniform to nearly one-hot rows."""
    cfg = synth.AttnConfig("kv8-scale", "bf16", 8, 2, 128, 16, 7200)
    wl, dv, orc = replay(cfg, [40, 1, 6], [300, 90, 333], 52)
    p = dv.prepare(wl.launches[0])
    dv.append(p)
    B.kv8_attention(p.info.kind, p.q, dv.k_cache, dv.v_cache, dv.scales, p.block_table, p.seq_lens,
                    p.cu, p.plan, p.info, p.ws, p.out, p.lse, scale=scale)
    torch.cuda.synchronize()
    orc.launch(wl.launches[0], attend=False)
    q, md = wl.launches[0].q.get().astype(np.float64), p.meta
    out, lse = paged_attention(q, orc.k_cache, orc.v_cache, md["block_table"], md["seq_lens"],
                               md["cu_seqlens_q"], 2, scale=scale)
    A, _ = paged_attention(q, orc.k_cache, np.abs(orc.v_cache), md["block_table"], md["seq_lens"],
                           md["cu_seqlens_q"], 2, scale=scale)
    ds = 132 * 2.0 ** -24 * scale * np.linalg.norm(q, axis=2).max() * \
        np.sqrt((orc.k_cache.astype(np.float64) ** 2).sum(3)).max()
    assert np.all(np.abs(p.out.double().cpu().numpy() - out)
                  <= 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 2 * ds + 2.0 ** -16) * A)
    assert np.all(np.abs(p.lse.double().cpu().numpy() - lse)
                  <= ds + 2.0 ** -16 * np.maximum(1, np.abs(lse)))


# rows merged from key-split tiles and from row items, joined ones, a shared
# prefix's chunks, whole tiles, two row items of one sequence
NAN = {
    "tiles": (8, 2, 128, [100], [2100], 0),
    "tiles-whole": (8, 2, 128, [100], [120], 0),
    "two-items": (16, 2, 64, [5] * 2, [1000, 2053], 0),
    "decode": (32, 8, 128, [1, 1], [1000, 257], 0),
    "decode-joined": (8, 2, 128, [1], [700], 0),
    "decode-short": (8, 2, 64, [1] * 5, [30, 1, 64, 65, 17], 0),
    "decode-shared": (8, 2, 128, [1] * 3, [2100, 2049, 2563], 2048),
    "decode-shared-tiles": (8, 2, 128, [1] * 3, [2100, 2049, 2563], 2048),
}


@pytest.mark.parametrize("where", ["query", "key", "value"])
@pytest.mark.parametrize("name", list(NAN))
def test_rows_without_a_number_stay_visible(name, where):
    """A row whose query, or a key it sees, is NaN comes out NaN (its log-sum-exp
    minus infinity) however its keys are split, one that sees a NaN value in that
    dim; no other row changes."""
    hq, hkv, d, q_lens, lens, prefix = NAN[name]
    cfg = synth.AttnConfig(f"kv8-nan-{name}", "bf16", hq, hkv, d, 16, 7300 + len(name))
    # a chip of 8 CUs: the shared keys are worth tiles of their own
    wl, dv, orc = replay(cfg, q_lens, lens, 53, prefix,
                         num_cus=8 if name == "decode-shared-tiles" else 0)
    ro = orc.launch(wl.launches[0])
    p = dv.prepare(wl.launches[0])
    assert name != "decode-shared-tiles" or p.info.n_shared_items > 0
    dv.append(p)
    dv.attend(p)
    torch.cuda.synchronize()
    plain, plain_lse = p.out.clone(), p.lse.clone()
    last = q_lens[0] - 1  # of the first sequence
    slot = int(p.slots[last])
    bad = torch.zeros(plain.shape, dtype=torch.bool, device="cuda")
    if where == "query":
        p.q[last, 1, 3] = float("nan")
        bad[last, 1] = True
    elif where == "key":
        dv.k_cache.view(torch.uint8)[slot // 16, 0, 0, slot % 16, 3] = 0x7F
        bad[last, :hq // hkv] = True
    else:
        dv.v_cache.view(torch.uint8)[slot // 16, 0, 5, slot % 16] = 0xFF
        bad[last, :hq // hkv, 5] = True
    dv.attend(p)
    torch.cuda.synchronize()
    keep = ~bad
    if where == "value":
        keep[:q_lens[0], :hq // hkv, 5] = False  # earlier tokens of the launch: either
        assert torch.equal(p.lse, plain_lse)
    else:
        assert torch.equal(p.lse == -float("inf"), bad.all(2))
        # a wavefront's reference moves for all its rows: each result is within 2^-16 of
        # itself (the head of this file), so two are within 2^-15
        ok = ~bad.all(2)
        assert torch.all((p.lse - plain_lse).abs()[ok] <= 2.0 ** -15 * plain_lse.abs().clamp(min=1)[ok])
    assert torch.isnan(p.out[bad]).all()
    # and the outputs are within the bound of the same exact ones
    md = ro["meta"]
    bo, _ = bounds(wl.launches[0].q.get().astype(np.float64), orc.k_cache, orc.v_cache,
                   md["block_table"], md["seq_lens"], md["cu_seqlens_q"], hkv, ro["out"], ro["lse"])
    diff = (p.out.double() - plain.double()).abs().cpu().numpy()
    assert np.all(diff[keep.cpu().numpy()] <= 2 * bo[keep.cpu().numpy()])


@pytest.mark.parametrize("where", ["key", "value"])
@pytest.mark.parametrize("hq, d, n, L", [(8, 128, 1, 700), (8, 64, 1, 9001), (16, 128, 5, 900),
                                         (16, 64, 5, 5000)])
def test_joined_wavefronts_keep_what_is_not_a_number(hq, d, n, L, where):
    """A NaN among keys whose weight underflows beside another wavefront's: the row is
    NaN, or its element is, as it is where one item holds all keys."""
    hkv = 2
    table, nb = tables([L], 12)
    c = Cache(nb, hkv, d, 12)
    mq = meta(table, [L], [n])
    kind = B.KIND_DECODE if n == 1 else B.KIND_VERIFY
    plan, info = B.plan(kind, n, mq[1], mq[2], hq, hkv, d, 16, B.PA_BF16_KV8, block_table=mq[0])
    from tests.test_capi_host import parse_plan
    rows = parse_plan(plan)[3]
    assert rows and all(t[7] & 2 for t in rows)  # every row item is one of a joined four
    ws = torch.empty(max(16, int(info.workspace_bytes)), dtype=torch.uint8, device="cuda")
    dm, dplan = [dev(x) for x in mq], dev(plan)
    q = torch.zeros((n, hq, d), dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 16.0
    out, lse = torch.empty_like(q), torch.empty((n, hq), device="cuda")
    r = np.random.default_rng(12)
    v = rows_of(r, L, hkv, d, "bf16")
    # a step's, a wavefront's and the item's ends; the last n tokens are not seen by all rows
    spots = sorted({0, 63, 191, 200, L // 3, L // 2, 3 * L // 4, L - n})
    for i, at in enumerate(spots):
        top = spots[(i + 1 + i % (len(spots) - 1)) % len(spots)]
        k = np.zeros((L, hkv, d), np.float32)
        k[top, :, 0] = 448.0  # its score lies above 600: 2^-900 for all others
        B.kv8_append(dev(k), dev(v), *[dev(x) for x in meta(table, [L], [L])], *c.args)
        blk, off = int(table[0, at // 16]), at % 16
        if where == "key":
            c.k.view(torch.uint8)[blk, 1, d // 64 - 1, off, 7] = 0x7F
        else:
            c.v.view(torch.uint8)[blk, 1, 9, off] = 0x7F
        B.kv8_attention(kind, q, *c.args, *dm, dplan, info, ws, out, lse)
        torch.cuda.synchronize()
        g = hq // hkv
        bad = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        bad[:, g:, slice(None) if where == "key" else 9] = True
        assert torch.equal(out.isnan(), bad), (at, top)
        assert torch.equal(lse == -float("inf"), bad.all(2)), (at, top)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_len", [1, 130])
def test_values_near_the_largest_stay_finite(d, q_len):
    """One key's probability lies 2^11 above the others', its values are 3e35:
    every sum stays in range."""
    L, at = 500, 300
    cfg = synth.AttnConfig(f"kv8-large-{d}", "bf16", 4, 2, d, 16, 7400 + d)
    wl, dv, _ = replay(cfg, [q_len], [L], 54)
    p = dv.prepare(wl.launches[0])
    table = p.meta["block_table"]
    k = np.zeros((L, 2, d), np.float32)
    v = np.zeros((L, 2, d), np.float32)
    k[at, :, 0] = 11 * 0.6931 * d ** 0.5 / 8
    v[at] = 3e35
    m = [dev(x) for x in meta(table, [L], [L])]
    B.kv8_append(dev(k), dev(v), *m, dv.k_cache, dv.v_cache, dv.scales)
    p.q.zero_()
    p.q[:, :, 0] = 8.0
    dv.attend(p)
    ko, vo = (torch.empty((L, 2, d), device="cuda") for _ in range(2))
    B.kv8_read(ko, vo, *m, dv.k_cache, dv.v_cache, dv.scales)
    torch.cuda.synchronize()
    w = np.exp(float(ko[at, 0, 0].double()) * 8 * d ** -0.5)
    val = float(vo[at, 0, 0].double())
    seen = np.arange(L - q_len + 1, L + 1).astype(float)
    ref = np.where(seen > at, w / (w + seen - 1), 0.0)[:, None, None]
    got = p.out.double().cpu().numpy() / val
    assert np.all(np.abs(got - ref) <= (2 * 2.0 ** -8 + 2.0 ** -12) * ref)


def test_decode_of_many_heads_without_workspace():
    """More than 32 heads per kv-head in a launch whose split row items would not
    fit the array of the call without workspace: tile items, streamed."""
    n, hq, hkv, d = 243, 128, 2, 128
    r = np.random.default_rng(8)
    lens = [513 + i % 11 for i in range(n)]
    table, nb = tables(lens, 8)
    c = Cache(nb, hkv, d, 8)
    # finite codes of ordinary scales everywhere
    for t in (c.k, c.v):
        u = t.view(torch.uint8)
        u.copy_(torch.where((u & 0x7F) == 0x7F, u & 0x87, u))
    c.scales.copy_(dev(r.integers(117, 120, c.scales.shape).astype(np.uint8)))
    m = meta(table, lens, [1] * n)
    plan, info = B.plan(B.KIND_DECODE, 1, m[1], m[2], hq, hkv, d, 16, B.PA_BF16_KV8,
                        block_table=m[0])
    assert info.n_tile_items > 0 and info.workspace_bytes <= B.NOALLOC_WORKSPACE_BYTES
    q = torch.randn((n, hq, d), device="cuda").to(torch.bfloat16)
    out = torch.empty_like(q)
    dm = [dev(x) for x in m]
    B.kv8_attention_decode_noalloc(q, *c.args, *dm, dev(plan), info, out)
    torch.cuda.synchronize()
    s = torch.exp2(c.scales.double() - 127)
    k = (c.k.double() * s[:, :, 0, None, None, None]).transpose(2, 3).reshape(nb, hkv, 16, d)
    v = (c.v.double() * s[:, :, 1, None, None]).transpose(2, 3)
    for i in range(0, n, 37):
        b = torch.from_numpy(table[i][table[i] >= 0]).cuda().long()
        kk = k[b].transpose(0, 1).reshape(hkv, -1, d)[:, :lens[i]]
        vv = v[b].transpose(0, 1).reshape(hkv, -1, d)[:, :lens[i]].contiguous()
        qq = q[i].double().view(hkv, hq // hkv, d)
        sc = torch.bmm(qq, kk.transpose(1, 2).contiguous()) * d ** -0.5
        pr = torch.softmax(sc, 2)
        ref = torch.bmm(pr, vv).view(hq, d)
        A = torch.bmm(pr, vv.abs()).view(hq, d)
        # scores' sums: (D + 4) 2^-24 scale |q| |k|, |q| of 128 normal values below 16
        ds = (d + 4) * 2.0 ** -24 * 16 * float(kk.norm(dim=2).max()) * d ** -0.5
        assert torch.all((out[i].double() - ref).abs()
                         <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2 * ds + 2.0 ** -16) * A)


@pytest.mark.parametrize("q_lens", [[1, 1, 1], [5, 5, 5], [40, 3, 100]])
def test_blocks_past_4_gib(q_lens):
    """The same launch on a small cache and on the last blocks of one whose keys and
    whose values pass 2^32 bytes: equal bit for bit."""
    hq, hkv, d = 16, 8, 128
    lens = [300, 77, 1100]
    far_nb = (1 << 32) // (hkv * 16 * d) + 2000
    table, nb = tables(lens, 11)
    r = np.random.default_rng(11)
    k, v = (dev(rows_of(r, sum(lens), hkv, d, "bf16"), torch.bfloat16) for _ in range(2))
    q = torch.randn((sum(q_lens), hq, d), device="cuda", generator=torch.Generator(
        "cuda").manual_seed(1)).to(torch.bfloat16)
    kind = {1: B.KIND_DECODE, 5: B.KIND_VERIFY}.get(q_lens[1], B.KIND_PREFILL)
    results = []
    for blocks, t in ((nb, table), (far_nb, np.where(table >= 0, table + far_nb - nb, -1))):
        ks, vs, ss = B.kv8_cache_shapes(blocks, hkv, d)
        cache = [torch.empty(ks, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn),
                 torch.empty(vs, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn),
                 torch.empty(ss, dtype=torch.uint8, device="cuda")]
        m = [dev(x) for x in meta(t, lens, lens)]
        B.kv8_append(k, v, *m, *cache)
        ko, vo = torch.empty_like(k), torch.empty_like(v)
        B.kv8_read(ko, vo, *m, *cache)
        mq = meta(t, lens, q_lens)
        plan, info = B.plan(kind, q_lens[0], mq[1], mq[2], hq, hkv, d, 16, B.PA_BF16_KV8,
                            block_table=mq[0])
        ws = torch.empty(max(16, int(info.workspace_bytes)), dtype=torch.uint8, device="cuda")
        out, lse = torch.empty_like(q), torch.empty((sum(q_lens), hq), device="cuda")
        B.kv8_attention(kind, q, *cache, *[dev(x) for x in mq], dev(plan), info, ws, out, lse)
        torch.cuda.synchronize()
        results.append((ko, vo, out, lse))
        del cache
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert torch.isfinite(results[0][2].float()).all()


@pytest.mark.parametrize("q_lens", [[40, 3], [1, 1]])
def test_odd_scales_array(q_lens):
    """One kv-head and an odd number of blocks: the last pair of scales shares its word
    with two bytes behind the array, which change nothing and stay as they are."""
    hq, hkv, d, lens = 4, 1, 128, [300, 77]
    table, nb = tables(lens, 14, spare=0)
    nb += 1 - nb % 2
    table[0, 3] = nb - 1  # the last block is in use
    r = np.random.default_rng(14)
    k, v = (dev(rows_of(r, sum(lens), hkv, d, "bf16"), torch.bfloat16) for _ in range(2))
    q = dev(rows_of(r, sum(q_lens), hq, d, "bf16"), torch.bfloat16)
    kind = B.KIND_DECODE if q_lens == [1, 1] else B.KIND_PREFILL
    m, mq = meta(table, lens, lens), meta(table, lens, q_lens)
    plan, info = B.plan(kind, 1, mq[1], mq[2], hq, hkv, d, 16, B.PA_BF16_KV8, block_table=mq[0])
    ws = torch.empty(max(16, int(info.workspace_bytes)), dtype=torch.uint8, device="cuda")
    results = []
    for behind in (0, 255):
        memory = torch.full((2 * nb + 2,), behind, dtype=torch.uint8, device="cuda")
        c = Cache(nb, hkv, d, 14)
        cache = c.k, c.v, memory[:2 * nb].view(nb, hkv, 2)
        B.kv8_append(k, v, *map(dev, m), *cache)
        out, lse = torch.empty_like(q), torch.empty((sum(q_lens), hq), device="cuda")
        B.kv8_attention(kind, q, *cache, *map(dev, mq), dev(plan), info, ws, out, lse)
        torch.cuda.synchronize()
        assert memory[2 * nb:].tolist() == [behind] * 2
        results.append((out, lse))
    assert torch.isfinite(results[0][0]).all()
    assert torch.equal(results[0][0], results[1][0]) and torch.equal(results[0][1], results[1][1])


# ---- norms and rotation -----------------------------------------------------------------------

ROPE = [
    # tokens, q heads, kv heads, head_dim, rot_dim, interleaved, norm, dtype, strided
    (1, 1, 1, 64, 64, False, True, "bf16", False),
    (3, 8, 2, 128, 128, False, True, "bf16", True),
    (5, 28, 4, 128, 64, True, True, "bf16", True),
    (70, 5, 1, 64, 32, False, True, "f32", True),
    (9, 4, 2, 64, 6, False, True, "f32", False),
    (9, 4, 2, 128, 6, True, True, "f32", True),
    (9, 3, 3, 128, 126, False, True, "bf16", False),
    (17, 4, 2, 128, 128, True, False, "f32", True),
    (17, 4, 2, 64, 0, False, True, "bf16", False),
    (257, 32, 8, 128, 128, False, True, "bf16", True),
    (13, 4, 0, 128, 128, False, True, "bf16", False),
    (13, 0, 3, 64, 48, False, True, "f32", False),
    (40, 64, 8, 64, 16, True, True, "bf16", True),
    # enough rows for two of them a lane, heads that do not fill the last wavefront
    (3600, 33, 4, 128, 128, False, True, "bf16", True),
    (7200, 33, 4, 64, 32, True, False, "bf16", False),
]


def rope_table(n, rot):
    freq = 1e4 ** (-np.arange(0, rot, 2) / max(rot, 1))
    a = np.arange(n)[:, None] * freq
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def rope_bound(x, y, table, weight, norm, interleaved, dtype):
    """Half a step of dtype, and (D + 11) 2^-24 of a pair's magnitudes, which bound
    both of its products."""
    half = table.shape[1] // 2
    z = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + 1e-6) if norm else x
    z = np.abs(z * (1 if weight is None or not norm else weight))
    mag = z.copy()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        s = z[..., a] + z[..., b]
        mag[..., a] = mag[..., b] = s
    eps = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    return eps * np.abs(y) + (x.shape[-1] + 11) * 2.0 ** -24 * mag + 1e-30


@pytest.mark.parametrize("case", range(len(ROPE)))
def test_norm_rope(case):
    T, hq, hkv, d, rot, inter, norm, dtype, wide = ROPE[case]
    say("[kv8] norm_rope", ROPE[case])
    r = np.random.default_rng(case)
    rnd = lambda *s: synth.round_to_dtype(  # noqa: E731
        (r.standard_normal(s) * np.exp(2 * r.standard_normal(s[:-1] + (1,)))).astype(np.float32), dtype)
    q, k = rnd(T, hq, d), rnd(T, hkv, d)
    if T > 5:
        q[2], k[3] = 0, 0  # rows of zeros: eps keeps them
    wq, wk = (synth.round_to_dtype(r.uniform(-2, 2, d).astype(np.float32), dtype) for _ in range(2))
    if case % 3 == 2:
        wq = None
    n_pos = 500
    table, pos = rope_table(n_pos, rot), r.integers(0, n_pos, T).astype(np.int32)
    skip = r.random(T) < 0.2 if T > 5 else np.zeros(T, bool)
    pos_in = pos.copy()
    pos_in[skip] = r.choice([-1, n_pos, 1 << 30, -(1 << 31)], skip.sum())
    t = DTYPE[dtype]
    put = (lambda x, i: strided(x, t, i)) if wide else (lambda x, i: dev(x, t))
    qo, ko = (torch.full((T, h, d), 7.0, dtype=t, device="cuda") for h in (hq, hkv))
    qd, kd = put(q, 0), put(k, 1)
    w = [None if x is None else dev(x, t) for x in (wq, wk)]
    B.qk_norm_rope(qd, kd, dev(pos_in), dev(table), qo, ko, *w, norm=norm, interleaved=inter)
    torch.cuda.synchronize()
    for x, o, wt in ((q, qo, wq), (k, ko, wk)):
        got = o.double().cpu().numpy()
        assert (got[skip] == 7).all()
        y = kv8.norm_rope(x, pos, table, wt, norm=norm, interleaved=inter)
        b = rope_bound(x.astype(np.float64), y, table, wt, norm, inter, dtype)
        assert np.all(np.abs(got - y)[~skip] <= b[~skip])
    if not wide:  # in place
        B.qk_norm_rope(qd, kd, dev(pos_in), dev(table), qd, kd, *w, norm=norm, interleaved=inter)
        torch.cuda.synchronize()
        keep = torch.from_numpy(~skip).cuda()
        assert torch.equal(qd[keep], qo[keep]) and torch.equal(kd[keep], ko[keep])
        assert torch.equal(qd[~keep], dev(q, t)[~keep])


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("d, rot, inter, dtype", [
    (128, 64, True, "bf16"), (128, 64, False, "bf16"), (64, 6, True, "f32"), (64, 6, False, "f32"),
    (64, 48, False, "f32"), (128, 126, True, "bf16"), (128, 0, False, "bf16"), (64, 0, True, "f32")])
def test_dims_that_are_not_turned_stay(d, rot, inter, dtype, norm):
    """Infinities, NaN and zeros of either sign behind rot_dim change no dim beside
    them; without norms those dims come out bit for bit."""
    T, hq, hkv, n_pos = 14, 5, 2, 50
    r = np.random.default_rng(d + rot)
    table, pos = rope_table(n_pos, rot), r.integers(1, n_pos, T).astype(np.int32)
    x = synth.round_to_dtype(r.standard_normal((T, hq + hkv, d)).astype(np.float32), dtype)
    special = [np.inf, -np.inf, np.nan, -0.0, 0.0]
    for t in range(T - 2):  # one or two of them in a head, beside ordinary values
        for h in range(hq + hkv):
            for _ in range(1 + (t + h) % 2):
                x[t, h, r.integers(rot, d)] = special[r.integers(5)]
    x[T - 2, :, rot:] = np.inf
    dt = DTYPE[dtype]
    q, k = dev(x[:, :hq], dt), dev(x[:, hq:], dt)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    B.qk_norm_rope(q, k, dev(pos), dev(table), qo, ko, norm=norm, interleaved=inter)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        y = kv8.norm_rope(x, pos, table, norm=norm, interleaved=inter)
        b = rope_bound(x.astype(np.float64), y, table, None, norm, inter, dtype)
    got = np.concatenate([qo.double().cpu().numpy(), ko.double().cpu().numpy()], 1)
    fin = np.isfinite(y)
    assert np.array_equal(got[~fin], y[~fin], equal_nan=True)
    assert np.all(np.abs(got - y)[fin] <= b[fin])
    if not norm:
        bits = torch.int16 if dtype == "bf16" else torch.int32
        for a, o in ((q, qo), (k, ko)):
            a, o = a[..., rot:].contiguous(), o[..., rot:].contiguous()
            same = (a.view(bits) == o.view(bits)) | (a.isnan() & o.isnan())
            assert same.all()


# ---- together ---------------------------------------------------------------------------------

class Chain:
    """A decode step of one layer, as a serving program runs it: norms and rotation
    of the projection's rows, append, attention, and the new tokens read back."""

    def __init__(self, lens, n_new, hq=8, hkv=2, d=128, seed=0):
        r = np.random.default_rng([seed, 4])
        self.hq, self.hkv, self.d, self.n_new = hq, hkv, d, n_new
        self.T = n_new * len(lens)
        self.lens = np.array(lens)
        self.table, nb = tables([x + n_new for x in lens], seed)
        self.cache = Cache(nb, hkv, d, seed)
        self.kc, self.vc = np.zeros((nb, hkv, 16, d)), np.zeros((nb, hkv, d, 16))
        self.ex = kv8.new_exponents(nb, hkv)
        n = int(self.lens.sum())
        k, v = rows_of(r, n, hkv, d, "bf16"), rows_of(r, n, hkv, d, "bf16")
        m = meta(self.table, lens, lens)
        kv8.append(self.kc, self.vc, self.ex, *m, k, v)
        B.kv8_append(dev(k, torch.bfloat16), dev(v, torch.bfloat16), *map(dev, m), *self.cache.args)
        self.m = meta(self.table, self.lens + n_new, [n_new] * len(lens))
        self.dm = [dev(x) for x in self.m]
        self.tab = rope_table(4096, d)
        self.pos = np.concatenate([np.arange(x, x + n_new) for x in lens]).astype(np.int32)
        self.w = [synth.round_to_dtype(r.uniform(0.5, 2, d).astype(np.float32), "bf16") for _ in range(2)]
        self.dw = [dev(x, torch.bfloat16) for x in self.w]
        self.dtab, self.dpos = dev(self.tab), dev(self.pos)
        self.qkv = torch.empty((self.T, hq + 2 * hkv, d), dtype=torch.bfloat16, device="cuda")
        self.q = torch.empty((self.T, hq, d), dtype=torch.bfloat16, device="cuda")
        self.k = torch.empty((self.T, hkv, d), dtype=torch.bfloat16, device="cuda")
        self.k_back, self.v_back = torch.empty_like(self.k), torch.empty_like(self.k)
        self.out = torch.empty_like(self.q)
        self.lse = torch.empty((self.T, hq), dtype=torch.float32, device="cuda")
        self.kind = B.KIND_DECODE if n_new == 1 else B.KIND_VERIFY
        plan, self.info = B.plan(self.kind, n_new, self.m[1], self.m[2], hq, hkv, d, 16,
                                 B.PA_BF16_KV8, block_table=self.m[0])
        self.plan = dev(plan)
        self.ws = torch.empty(max(16, int(self.info.workspace_bytes)), dtype=torch.uint8, device="cuda")

    def feed(self, seed):
        r = np.random.default_rng([seed, 5])
        self.x = rows_of(r, self.T, self.hq + 2 * self.hkv, self.d, "bf16")
        self.qkv.copy_(dev(self.x, torch.bfloat16))

    def step(self, stream=None):
        hq, hkv = self.hq, self.hkv
        B.qk_norm_rope(self.qkv[:, :hq], self.qkv[:, hq:hq + hkv], self.dpos, self.dtab, self.q,
                       self.k, *self.dw, stream=stream)
        B.kv8_append(self.k, self.qkv[:, hq + hkv:], *self.dm, *self.cache.args, stream=stream)
        B.kv8_attention(self.kind, self.q, *self.cache.args, *self.dm, self.plan, self.info, self.ws,
                        self.out, self.lse, stream=stream)
        B.kv8_read(self.k_back, self.v_back, *self.dm, *self.cache.args, stream=stream)

    def check(self, label):
        """The rotated rows against the oracle's, then everything after them from the
        device's own rows (their rounding is checked, not carried along)."""
        hq, hkv = self.hq, self.hkv
        for x, got, w in ((self.x[:, :hq], self.q, self.w[0]), (self.x[:, hq:hq + hkv], self.k, self.w[1])):
            y = kv8.norm_rope(x, self.pos, self.tab, w)
            b = rope_bound(x.astype(np.float64), y, self.tab, w, True, False, "bf16")
            assert np.all(np.abs(got.double().cpu().numpy() - y) <= b), label
        kv8.append(self.kc, self.vc, self.ex, *self.m, self.k.double().cpu().numpy(),
                   self.x[:, hq + hkv:])
        seq = np.repeat(np.arange(len(self.lens)), self.n_new)
        blk, off = self.table[seq, self.pos // 16], self.pos % 16
        assert np.array_equal(self.k_back.double().cpu().numpy(), self.kc[blk, :, off]), label
        assert np.array_equal(self.v_back.double().cpu().numpy(), self.vc[blk, :, :, off]), label
        q = self.q.double().cpu().numpy()
        ro, rl = paged_attention(q, self.kc, self.vc, *self.m, hkv)
        bo, bl = bounds(q, self.kc, self.vc, *self.m, hkv, ro, rl)
        eo = np.abs(self.out.double().cpu().numpy() - ro)
        el = np.abs(self.lse.double().cpu().numpy() - rl)
        say(f"[kv8] {label}: worst out {np.max(eo / bo):.2f}, lse {np.max(el / bl):.2f} of the bound")
        assert np.all(eo <= bo) and np.all(el <= bl), label


@pytest.mark.parametrize("n_new", [1, 4])
def test_step(n_new):
    c = Chain([100, 15, 16, 700, 33], n_new)
    for i in range(3):  # the same positions again: the scales only grow
        c.feed(i)
        c.step()
        torch.cuda.synchronize()
        c.check(f"step {n_new} {i}")


def test_step_on_another_stream():
    c = Chain([100, 15, 700], 1, seed=1)
    c.feed(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.step(stream=side)
    side.synchronize()
    c.check("side stream argument")
    c.feed(1)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.step()
    side.synchronize()
    c.check("side stream as current")


def test_captured_step():
    """A captured step replayed with other inputs between, eager work beside it."""
    c = Chain([100, 15, 700, 2000], 1, hq=16, seed=2)
    c.feed(0)
    c.step()  # modules are loaded outside the capture
    torch.cuda.synchronize()
    c.check("before the capture")
    g = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
        c.step()
    torch.cuda.current_stream().wait_stream(side)
    for i in range(4):
        c.feed(10 + i)
        c.out.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        c.check(f"replay {i}")
        if i == 1:
            c.feed(20)
            c.step()
            torch.cuda.synchronize()
            c.check("eager between replays")


def test_workload_steps():
    """Workloads of the framework on an 8-bit cache: prefix hits, chunks, drafts
    rolled back, several launches, through the staged path."""
    from paper_2605_11232_amd.runtime import DeviceReplay, Staging, plan_words_bound
    for name, scale in (("prefill", 0.05), ("decode", 0.04), ("mixed", 0.03), ("verify", 0.06)):
        wl = synth.workload(name, scale=scale, steps=2)
        cfg = wl.cfg
        dv, orc = DeviceReplay(wl, kv8=True).setup(), OracleReplay(wl, kv8=True).setup()
        launches = list(wl.launches[:2]) + ([wl.step(1)] if wl.step else [])
        n, T = max(len(x.seq_ids) for x in launches), max(x.total_q for x in launches)
        st = [Staging(dv.device, n, wl.max_blocks_per_seq, T,
                      plan_words_bound(cfg, n, T, wl.max_blocks_per_seq)) for _ in range(2)]
        for i, ln in enumerate(launches):
            rows = sorted({(int(t), int(h)) for t, h in zip(
                np.random.default_rng(i).integers(0, ln.total_q, 60),
                np.random.default_rng(i + 9).integers(0, cfg.num_q_heads, 60))})
            ro = orc.launch(ln, rows=rows)
            x = [torch.from_numpy(a.get()).to("cuda", torch.bfloat16) for a in (ln.q, ln.k_new, ln.v_new)]
            out = torch.empty((ln.total_q, cfg.num_q_heads, cfg.head_dim), dtype=torch.bfloat16,
                              device="cuda")
            lse = torch.empty((ln.total_q, cfg.num_q_heads), dtype=torch.float32, device="cuda")
            p = dv.prepare_staged(ln, st[i % 2], *x, out, lse)
            dv.append(p)
            dv.attend(p)
            torch.cuda.synchronize()
            t, h = np.array(rows).T
            A, _ = paged_attention(ln.q.get().astype(np.float64), orc.k_cache, np.abs(orc.v_cache),
                                   ro["meta"]["block_table"], ro["meta"]["seq_lens"],
                                   ro["meta"]["cu_seqlens_q"], cfg.num_kv_heads, rows=rows)
            err = np.abs(out.double().cpu().numpy() - ro["out"])[t, h]
            # |q| |k| / sqrt(D) of normal values is below 40: 2 ds < 2^-10
            b = 2.0 ** -8 * np.abs(ro["out"][t, h]) + (2.0 ** -8 + 2.0 ** -10) * A[t, h]
            say(f"[kv8] {name} launch {i}: worst {np.max(err / b):.2f} of the bound")
            assert np.all(err <= b)
            assert np.all(np.abs(lse.double().cpu().numpy() - ro["lse"])[t, h] <= 2.0 ** -10)
            orc.finish(ln)
            dv.finish(ln, batched=True)
