"""GPU parity of the 4-bit cache (append, read back, attention) against the float64
oracle, at the sizes, masks and values where they can go wrong.

Bounds.  Append and read back: exact, codes and scales bit for bit.  Attention over the
cache's values: as over the 8-bit cache (the head of tests/test_gpu_kv8.py): a probability
times its token's scale, a power of two, is rounded to bf16 as the probability alone would
be."""
import numpy as np
import pytest
import torch

from oracle import kv4
from oracle.attention import paged_attention
from oracle.run import OracleReplay
from paper_2605_11232_amd import binding as B, synth
from tests.parity import say
from tests.test_gpu_kv8 import (APPENDS, ATTN, DTYPE, NAN, bounds, check, dev, meta, rows_of,
                                strided, tables)
from tests.test_gpu_paths import launch_workload

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def split(byte_array):
    """Codes of packed bytes, low halves first."""
    return np.stack([byte_array & 15, byte_array >> 4], -1).reshape(*byte_array.shape[:-1], -1)


class Cache:
    """A device cache whose every byte starts at random (NaN scales among them)."""

    def __init__(self, nb, hkv, d, seed=0):
        r = np.random.default_rng([seed, 9])
        self.nb, self.hkv, self.d = nb, hkv, d
        self.args = tuple(torch.from_numpy(r.integers(0, 256, s, dtype=np.uint8)).cuda()
                          for s in B.kv4_cache_shapes(nb, hkv, d))
        self.k, self.v, self.scales = self.args

    def raw(self):
        """Codes of keys and values as [NB, Hkv, 16, D], scale bytes [NB, Hkv, 16, D / 32 + 1]."""
        k, v, s = (x.cpu().numpy() for x in self.args)
        v = split(v.reshape(self.nb, self.hkv, self.d // 32, 16, 2, 8))  # [.., c, i, a, token]
        v = v.transpose(0, 1, 5, 2, 4, 3).reshape(self.nb, self.hkv, 16, self.d)
        return split(k), v, s.transpose(0, 1, 3, 2)

    def values(self):
        """Keys [NB, Hkv, 16, D] and values [NB, Hkv, D, 16] in float64."""
        k, v, s = self.raw()
        k = kv4.values(k.reshape(*k.shape[:3], -1, 32), s[..., :-1]).reshape(k.shape)
        return k, kv4.values(v, s[..., -1]).transpose(0, 1, 3, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(APPENDS))
def test_append_and_read(name, dtype):
    """Codes, scales and untouched halves of bytes after every append, and the rows read
    back."""
    say("[kv4] append", name, dtype)
    hkv, d, steps = APPENDS[name]
    r = np.random.default_rng(len(name))
    table, nb = tables(steps[-1][0], 5)
    c = Cache(nb, hkv, d)
    k_ref, v_ref, s_ref = (x.copy() for x in c.raw())
    for lens, q in steps:
        T = sum(q)
        k, v = rows_of(r, T, hkv, d, dtype), rows_of(r, T, hkv, d, dtype)
        m = meta(table, lens, q)
        seq = np.repeat(np.arange(len(q)), q)
        pos = np.concatenate([np.arange(L - x, L) for L, x in zip(lens, q)] or [[]]).astype(int)
        blk, off = table[seq, pos // 16], pos % 16
        kq, ks = kv4.quantise(k.reshape(T, hkv, d // 32, 32))
        vq, vs = kv4.quantise(v)
        k_ref[blk, :, off], v_ref[blk, :, off] = kq.reshape(T, hkv, d), vq
        s_ref[blk, :, off] = np.concatenate([ks, vs[..., None]], -1)
        B.kv4_append(strided(k, DTYPE[dtype], 0), strided(v, DTYPE[dtype], 2), *map(dev, m), *c.args)
        torch.cuda.synchronize()
        for got, want in zip(c.raw(), (k_ref, v_ref, s_ref)):
            assert np.array_equal(got, want)
        kc, vc = c.values()
        for n in (q, lens):  # this step's rows, then whole contexts, packed and strided
            rows = sum(n)
            mm = meta(table, lens, n)
            ko = torch.full((rows + 2, hkv, d), 7.0, dtype=DTYPE[dtype], device="cuda")
            wide = torch.full((rows, 2 * hkv, d), 7.0, dtype=DTYPE[dtype], device="cuda")
            B.kv4_read(ko[:rows], wide[:, hkv:], *map(dev, mm), *c.args)
            torch.cuda.synchronize()
            seq = np.repeat(np.arange(len(n)), n)
            pos = np.concatenate([np.arange(L - x, L) for L, x in zip(lens, n)] or [[]]).astype(int)
            blk = table[seq, pos // 16]
            assert np.array_equal(ko[:rows].double().cpu().numpy(), kc[blk, :, pos % 16])
            assert np.array_equal(wide[:, hkv:].double().cpu().numpy(), vc[blk, :, :, pos % 16])
            assert (ko[rows:] == 7).all() and (wide[:, :hkv] == 7).all()


@pytest.mark.parametrize("d", [64, 128])
def test_append_of_values_at_the_ends_of_the_range(d):
    """Zeros of either sign, ties, magnitudes below the smallest and above the largest code,
    and values that are not finite, which make their 32 dims, or the whole value, NaN."""
    hkv, r = 2, np.random.default_rng(d)
    tops = [0.0, -0.0, 2.0 ** -126, 1e-40, 3.3e38, 7 * 2.0 ** 100, 7.5 * 2.0 ** 100, 7.0,
            np.nextafter(np.float32(7), np.float32(8)), 6.0, 3.5, 1e-30, 1e30, np.inf, -np.inf, np.nan]
    T = len(tops)
    x = np.stack([np.full((hkv, d), t) for t in tops])
    ties = np.array([1, 0.5, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 0.1]) / 7
    x[:, :, 1:] *= r.choice(np.concatenate([ties, -ties]), (T, hkv, d - 1))
    x[:13, :, d // 2] = 0.0
    x[13:] = r.standard_normal((3, hkv, d))  # one dim that is not finite among others
    x[13:, 1, 37] = tops[13:]
    x = x.astype(np.float32)
    with np.errstate(invalid="ignore"):
        kq, ks = kv4.quantise(x.reshape(T, hkv, d // 32, 32))
        vq, vs = kv4.quantise(-x)
    table, nb = tables([T], 6)
    c = Cache(nb, hkv, d, 1)
    m = meta(table, [T], [T])
    B.kv4_append(dev(x), dev(-x), *map(dev, m), *c.args)
    ko, vo = (torch.empty((T, hkv, d), device="cuda") for _ in range(2))
    B.kv4_read(ko, vo, *map(dev, m), *c.args)
    torch.cuda.synchronize()
    k, v, s = (a[table[0, 0]].swapaxes(0, 1) for a in c.raw())
    assert np.array_equal(s[..., :-1], ks) and np.array_equal(s[..., -1], vs)
    assert np.array_equal(k, kq.reshape(k.shape)) and np.array_equal(v, vq)
    want = kv4.values(kq, ks).reshape(x.shape), kv4.values(vq, vs)
    for got, ref in zip((ko, vo), want):
        got = got.double().cpu().numpy()
        assert np.array_equal(got, ref, equal_nan=True)
        assert np.array_equal(np.signbit(got[:13]), np.signbit(ref[:13]))
    assert np.isnan(want[0][13:, 1, 32:64]).all() and np.isfinite(want[0][13:, 1, :32]).all()
    assert np.isnan(want[1][13:, 1]).all() and np.isfinite(want[1][13:, 0]).all()


def test_append_skips_what_it_cannot_place():
    """Block ids outside the cache, positions past the table and rows past the caller's
    write nothing; the other sequences are stored."""
    hkv, d = 2, 128
    lens, q = [20, 40, 18], [20, 4, 2]
    table, nb = tables(lens, 7)
    c, want = Cache(nb, hkv, d, 2), Cache(nb, hkv, d, 2)
    r = np.random.default_rng(3)
    k, v = (dev(rows_of(r, sum(q), hkv, d, "bf16"), torch.bfloat16) for _ in range(2))
    m = meta(table, lens, q)
    B.kv4_append(k[20:24], v[20:24], *map(dev, meta(table[1:2], [40], [4])), *want.args)
    bad = m[0].copy()
    bad[0, 0], bad[0, 1], bad[2, 1] = -1, nb, -7
    B.kv4_append(k, v, dev(bad), dev(m[1]), dev(m[2]), *c.args)
    out = torch.full((2, sum(q), hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
    B.kv4_read(out[0], out[1], dev(bad), dev(m[1]), dev(m[2]), *c.args)
    torch.cuda.synchronize()
    assert all(np.array_equal(a, b) for a, b in zip(c.raw(), want.raw()))
    assert (out[:, :20] == 7).all() and (out[:, 24:] == 7).all() and (out[:, 20:24] != 7).any()
    # a table of two columns: the second sequence's last tokens are past it; a row count of
    # 22: the third sequence's rows are past it; more rows than positions
    c, want = Cache(nb, hkv, d, 2), Cache(nb, hkv, d, 2)
    B.kv4_append(k[:20], v[:20], *map(dev, meta(table[:1], [20], [20])), *want.args)
    two = np.ascontiguousarray(m[0][:, :2])
    B.kv4_append(k[:22], v[:22], dev(two), dev(m[1]), dev(m[2]), *c.args)
    B.kv4_append(k, v, dev(m[0]), dev(np.array([3, 3, 1], np.int32)), dev(m[2]), *c.args)
    torch.cuda.synchronize()
    assert all(np.array_equal(x, y) for x, y in zip(c.raw(), want.raw()))


# ---- attention --------------------------------------------------------------------------------

def replay(cfg, q_lens, lens, seed, prefix=0, num_cus=0):
    from paper_2605_11232_amd.runtime import DeviceReplay
    wl = launch_workload(cfg, q_lens, lens, seed, prefix)
    dv = DeviceReplay(wl, kv4=True, num_cus=num_cus)
    # unwritten slots: the largest codes under NaN scales
    for t in (dv.k_cache, dv.v_cache, dv.scales):
        t.fill_(255)
    return wl, dv.setup(), OracleReplay(wl, kv4=True).setup()


def attention_case(name, num_cus=0):
    hq, hkv, d, q_lens, lens, prefix = ATTN[name]
    say("[kv4] attention", name)
    cfg = synth.AttnConfig(f"kv4-{name}", "bf16", hq, hkv, d, 16, 8000 + len(name))
    wl, dv, orc = replay(cfg, q_lens, lens, 60, prefix, num_cus=num_cus)
    ro = orc.launch(wl.launches[0])
    p = dv.run(wl.launches[0])
    torch.cuda.synchronize()
    assert p.info.dtype == B.PA_BF16_KV4
    check(p, wl.launches[0].q.get().astype(np.float64), orc, ro, hkv, name)
    first = p.out.clone(), p.lse.clone()
    p.out.fill_(3.0), p.lse.fill_(3.0)
    dv.attend(p)  # the plan's counters are as they were
    torch.cuda.synchronize()
    assert torch.equal(p.out, first[0]) and torch.equal(p.lse, first[1])
    if p.kind == "decode" and p.info.workspace_bytes <= B.NOALLOC_WORKSPACE_BYTES:
        out, lse = torch.empty_like(p.out), torch.empty_like(p.lse)
        B.kv4_attention_decode_noalloc(p.q, dv.k_cache, dv.v_cache, dv.scales, p.block_table,
                                       p.seq_lens, p.cu, p.plan, p.info, out, lse)
        torch.cuda.synchronize()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    return p.info


@pytest.mark.parametrize("name", list(ATTN))
def test_attention(name):
    attention_case(name)


@pytest.mark.parametrize("name", ["shared", "shared-64", "verify-shared"])
def test_attention_on_a_split_off_prefix(name):
    """The same launches planned for a chip so small that the shared keys are worth
    tiles of their own."""
    assert attention_case(name, num_cus=8).n_shared_items > 0


def test_attention_with_tail_lists():
    """A launch with more tiles than the chip holds at once: wildcard workgroups take the
    last ones."""
    cfg = synth.AttnConfig("kv4-tail-lists", "bf16", 16, 8, 64, 16, 8100)
    wl, dv, orc = replay(cfg, [520] * 12, [520] * 12, 61)
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


@pytest.mark.parametrize("scale", [1e-3, 1.0, 3.0])
def test_attention_scale(scale):
    """The caller's softmax scale, from nearly uniform to nearly one-hot rows."""
    cfg = synth.AttnConfig("kv4-scale", "bf16", 8, 2, 128, 16, 8200)
    wl, dv, orc = replay(cfg, [40, 1, 6], [300, 90, 333], 62)
    p = dv.prepare(wl.launches[0])
    dv.append(p)
    B.kv4_attention(p.info.kind, p.q, dv.k_cache, dv.v_cache, dv.scales, p.block_table, p.seq_lens,
                    p.cu, p.plan, p.info, p.ws, p.out, p.lse, scale=scale)
    torch.cuda.synchronize()
    orc.launch(wl.launches[0], attend=False)
    q, md = wl.launches[0].q.get().astype(np.float64), p.meta
    where = md["block_table"], md["seq_lens"], md["cu_seqlens_q"], 2
    out, lse = paged_attention(q, orc.k_cache, orc.v_cache, *where, scale=scale)
    A, _ = paged_attention(q, orc.k_cache, np.abs(orc.v_cache), *where, scale=scale)
    ds = 132 * 2.0 ** -24 * scale * np.linalg.norm(q, axis=2).max() * \
        np.sqrt((orc.k_cache.astype(np.float64) ** 2).sum(3)).max()
    assert np.all(np.abs(p.out.double().cpu().numpy() - out)
                  <= 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 2 * ds + 2.0 ** -16) * A)
    assert np.all(np.abs(p.lse.double().cpu().numpy() - lse)
                  <= ds + 2.0 ** -16 * np.maximum(1, np.abs(lse)))


@pytest.mark.parametrize("where", ["query", "key", "value"])
@pytest.mark.parametrize("name", list(NAN))
def test_rows_without_a_number_stay_visible(name, where):
    """A row whose query, or a key or value it sees, is NaN comes out NaN however its keys
    are split (for a query or key its log-sum-exp is minus infinity); no other row changes,
    earlier tokens of the launch among them."""
    hq, hkv, d, q_lens, lens, prefix = NAN[name]
    cfg = synth.AttnConfig(f"kv4-nan-{name}", "bf16", hq, hkv, d, 16, 8300 + len(name))
    # a chip of 8 CUs: the shared keys are worth tiles of their own
    wl, dv, orc = replay(cfg, q_lens, lens, 63, prefix,
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
    else:  # a token stored with a NaN in one dim
        seq = [t[:1] for t in (p.block_table, p.seq_lens)]
        cu = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
        k, v = p.k_new[last:last + 1].clone(), p.v_new[last:last + 1].clone()
        (k if where == "key" else v)[0, 0, 5] = float("nan")
        B.kv4_append(k, v, *seq, cu, dv.k_cache, dv.v_cache, dv.scales)
        bad[last, :hq // hkv] = True
    dv.attend(p)
    torch.cuda.synchronize()
    assert torch.equal(p.out.isnan(), bad)
    ok = ~bad.all(2)
    if where == "value":
        assert torch.equal(p.lse, plain_lse)
    else:
        assert torch.equal(p.lse == -float("inf"), ~ok)
        # a wavefront's reference moves for all its rows: each result is within 2^-16 of
        # itself, so two are within 2^-15
        assert torch.all((p.lse - plain_lse).abs()[ok] <= 2.0 ** -15 * plain_lse.abs().clamp(min=1)[ok])
    md = ro["meta"]
    bo, _ = bounds(wl.launches[0].q.get().astype(np.float64), orc.k_cache, orc.v_cache,
                   md["block_table"], md["seq_lens"], md["cu_seqlens_q"], hkv, ro["out"], ro["lse"])
    diff = (p.out.double() - plain.double()).abs().cpu().numpy()
    keep = (~bad).cpu().numpy()
    assert np.all(diff[keep] <= 2 * bo[keep])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_len", [1, 130])
def test_values_of_the_largest_scale_stay_finite(d, q_len):
    """One key's probability lies 2^11 above the others', all values are 6 * 2^100: every
    sum stays in range."""
    L, at = 500, 300
    cfg = synth.AttnConfig(f"kv4-large-{d}", "bf16", 4, 2, d, 16, 8400 + d)
    wl, dv, _ = replay(cfg, [q_len], [L], 64)
    p = dv.prepare(wl.launches[0])
    k, v = np.zeros((L, 2, d), np.float32), np.full((L, 2, d), 3e38, np.float32)
    v[::2] *= -1
    k[at, :, 0] = 11 * 0.6931 * d ** 0.5 / 8
    m = [dev(x) for x in meta(p.meta["block_table"], [L], [L])]
    B.kv4_append(dev(k), dev(v), *m, dv.k_cache, dv.v_cache, dv.scales)
    p.q.zero_()
    p.q[:, :, 0] = 8.0
    dv.attend(p)
    ko = torch.empty((L, 2, d), device="cuda")
    B.kv4_read(ko, torch.empty_like(ko), *m, dv.k_cache, dv.v_cache, dv.scales)
    torch.cuda.synchronize()
    w = np.exp(float(ko[at, 0, 0].double()) * 8 * d ** -0.5)
    ref, size = [], []
    for n in range(L - q_len + 1, L + 1):
        p_t = np.ones(n)
        if n > at:
            p_t[at] = w
        sign = np.where(np.arange(n) % 2, 1.0, -1.0)
        ref.append((p_t * sign).sum() / p_t.sum())
    got = p.out.double().cpu().numpy() / (6 * 2.0 ** 100)
    assert np.all(np.abs(got - np.array(ref)[:, None, None])
                  <= 2.0 ** -8 * np.abs(np.array(ref))[:, None, None] + 2.0 ** -8 + 2.0 ** -12)


@pytest.mark.parametrize("q_lens", [[1, 1, 1], [5, 5, 5], [40, 3, 100]])
def test_blocks_past_4_gib(q_lens):
    """The same launch on a small cache and on the last blocks of one whose keys and whose
    values pass 2^32 bytes: equal bit for bit."""
    hq, hkv, d = 16, 8, 128
    lens = [300, 77, 1100]
    far_nb = (1 << 32) // (hkv * 8 * d) + 2000
    table, nb = tables(lens, 11)
    r = np.random.default_rng(11)
    k, v = (dev(rows_of(r, sum(lens), hkv, d, "bf16"), torch.bfloat16) for _ in range(2))
    q = torch.randn((sum(q_lens), hq, d), device="cuda", generator=torch.Generator(
        "cuda").manual_seed(1)).to(torch.bfloat16)
    kind = {1: B.KIND_DECODE, 5: B.KIND_VERIFY}.get(q_lens[1], B.KIND_PREFILL)
    results = []
    for blocks, t in ((nb, table), (far_nb, np.where(table >= 0, table + far_nb - nb, -1))):
        cache = [torch.empty(s, dtype=torch.uint8, device="cuda")
                 for s in B.kv4_cache_shapes(blocks, hkv, d)]
        m = [dev(x) for x in meta(t, lens, lens)]
        B.kv4_append(k, v, *m, *cache)
        ko, vo = torch.empty_like(k), torch.empty_like(v)
        B.kv4_read(ko, vo, *m, *cache)
        mq = meta(t, lens, q_lens)
        plan, info = B.plan(kind, q_lens[0], mq[1], mq[2], hq, hkv, d, 16, B.PA_BF16_KV4,
                            block_table=mq[0])
        ws = torch.empty(max(16, int(info.workspace_bytes)), dtype=torch.uint8, device="cuda")
        out, lse = torch.empty_like(q), torch.empty((sum(q_lens), hq), device="cuda")
        B.kv4_attention(kind, q, *cache, *[dev(x) for x in mq], dev(plan), info, ws, out, lse)
        torch.cuda.synchronize()
        results.append((ko, vo, out, lse))
        del cache
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert torch.isfinite(results[0][2].float()).all()


# ---- together ---------------------------------------------------------------------------------

class Step:
    """A decode or verification step of one layer: append, attention, the new tokens read
    back."""

    def __init__(self, lens, n_new, hq=8, hkv=2, d=128, seed=0):
        r = np.random.default_rng([seed, 4])
        self.hq, self.hkv, self.d, self.T = hq, hkv, d, n_new * len(lens)
        lens = np.array(lens)
        self.table, nb = tables(lens + n_new, seed)
        self.cache = Cache(nb, hkv, d, seed)
        n = int(lens.sum())
        k, v = rows_of(r, n, hkv, d, "bf16"), rows_of(r, n, hkv, d, "bf16")
        m = meta(self.table, lens, lens)
        B.kv4_append(dev(k, torch.bfloat16), dev(v, torch.bfloat16), *map(dev, m), *self.cache.args)
        self.m = meta(self.table, lens + n_new, [n_new] * len(lens))
        self.dm = [dev(x) for x in self.m]
        seq = np.repeat(np.arange(len(lens)), n_new)
        self.at = seq, np.concatenate([np.arange(x, x + n_new) for x in lens])
        self.q = torch.empty((self.T, hq, d), dtype=torch.bfloat16, device="cuda")
        self.k = torch.empty((self.T, hkv, d), dtype=torch.bfloat16, device="cuda")
        self.v, self.k_back, self.v_back = (torch.empty_like(self.k) for _ in range(3))
        self.out, self.lse = torch.empty_like(self.q), torch.empty((self.T, hq), device="cuda")
        self.kind = B.KIND_DECODE if n_new == 1 else B.KIND_VERIFY
        plan, self.info = B.plan(self.kind, n_new, self.m[1], self.m[2], hq, hkv, d, 16,
                                 B.PA_BF16_KV4, block_table=self.m[0])
        self.plan = dev(plan)
        self.ws = torch.empty(max(16, int(self.info.workspace_bytes)), dtype=torch.uint8, device="cuda")

    def feed(self, seed):
        r = np.random.default_rng([seed, 5])
        for x, h in ((self.q, self.hq), (self.k, self.hkv), (self.v, self.hkv)):
            x.copy_(dev(rows_of(r, self.T, h, self.d, "bf16"), torch.bfloat16))

    def step(self, stream=None):
        B.kv4_append(self.k, self.v, *self.dm, *self.cache.args, stream=stream)
        B.kv4_attention(self.kind, self.q, *self.cache.args, *self.dm, self.plan, self.info, self.ws,
                        self.out, self.lse, stream=stream)
        B.kv4_read(self.k_back, self.v_back, *self.dm, *self.cache.args, stream=stream)

    def check(self, label):
        kc, vc = self.cache.values()  # unwritten slots among them: looked at nowhere below
        k, v = self.k.double().cpu().numpy(), self.v.double().cpu().numpy()
        assert np.array_equal(self.k_back.double().cpu().numpy(), kv4.round_keys(k)), label
        assert np.array_equal(self.v_back.double().cpu().numpy(), kv4.round_values(v)), label
        seq, pos = self.at
        blk = self.table[seq, pos // 16]
        assert np.array_equal(kc[blk, :, pos % 16], kv4.round_keys(k)), label
        q = self.q.double().cpu().numpy()
        used = np.zeros(kc.shape[:1] + (16,), bool)
        for row, L in zip(self.table, self.m[1]):
            t = np.arange(L)
            used[row[t // 16], t % 16] = True
        kc, vc = np.where(used[:, None, :, None], kc, 0), np.where(used[:, None, None], vc, 0)
        ro, rl = paged_attention(q, kc, vc, *self.m, self.hkv)
        bo, bl = bounds(q, kc, vc, *self.m, self.hkv, ro, rl)
        eo = np.abs(self.out.double().cpu().numpy() - ro)
        el = np.abs(self.lse.double().cpu().numpy() - rl)
        # Probabilities below 2^-126 of a row's largest, and their products with a value's scale,
        # are zero in float32 and bf16: each then takes less than 2^-126 |v| from the sum, or
        # 2^-126 times a code of at most 6.  (Codes of zero leave dims whose other terms are all
        # of that kind.)
        bo = bo + int(self.m[1].max()) * 2.0 ** -126 * max(6.0, np.abs(vc).max())
        say(f"[kv4] {label}: worst out {np.max(eo / bo):.2f}, lse {np.max(el / bl):.2f} of the bound")
        assert np.all(eo <= bo) and np.all(el <= bl), label


@pytest.mark.parametrize("n_new, d", [(1, 128), (4, 128), (5, 64)])
def test_step(n_new, d):
    c = Step([100, 15, 16, 700, 33], n_new, d=d)
    for i in range(3):  # the same positions again
        c.feed(i)
        c.step()
        torch.cuda.synchronize()
        c.check(f"step {n_new} {i}")


def test_step_on_another_stream():
    c = Step([100, 15, 700], 1, seed=1)
    side = torch.cuda.Stream()
    for i in range(2):
        c.feed(i)
        side.wait_stream(torch.cuda.current_stream())
        if i == 0:
            c.step(stream=side)
        else:
            with torch.cuda.stream(side):
                c.step()
        side.synchronize()
        c.check(f"side stream {i}")


def test_captured_step():
    """A captured step replayed with other inputs between, eager work beside it."""
    c = Step([100, 15, 700, 2000], 1, hq=16, seed=2)
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
    """Workloads of the framework on a 4-bit cache: prefix hits, chunks, drafts rolled back,
    several launches, through the staged path."""
    from paper_2605_11232_amd.runtime import DeviceReplay, Staging, plan_words_bound
    for name, scale in (("prefill", 0.05), ("decode", 0.04), ("mixed", 0.03), ("verify", 0.06)):
        wl = synth.workload(name, scale=scale, steps=2)
        cfg = wl.cfg
        dv, orc = DeviceReplay(wl, kv4=True).setup(), OracleReplay(wl, kv4=True).setup()
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
            say(f"[kv4] {name} launch {i}: worst {np.max(err / b):.2f} of the bound")
            assert np.all(err <= b)
            assert np.all(np.abs(lse.double().cpu().numpy() - ro["lse"])[t, h] <= 2.0 ** -10)
            orc.finish(ln)
            dv.finish(ln, batched=True)
