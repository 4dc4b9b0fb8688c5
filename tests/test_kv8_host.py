"""The 8-bit cache on the host: the oracle's rounding against torch's e4m3 and
brute force, plans for it, and every refusal of its entry points (made before
anything is launched: the pointers below are never read)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2605_11232_amd import binding as B, synth
from paper_2605_11232_amd.runtime import plan_words_bound


def e4m3_values():
    """All finite non-negative e4m3 numbers, by their bits."""
    out = []
    for code in range(0x7F):
        x, m = code >> 3, code & 7
        out.append((8 + m) * 2.0 ** (x - 10) if x else m * 2.0 ** -9)
    return np.array(out)


def test_oracle_rounding_is_nearest_even():
    v = e4m3_values()
    assert v[-1] == 448 and len(set(v)) == 127
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9),
                        np.random.default_rng(1).uniform(0, 448, 2000),
                        2.0 ** np.random.default_rng(2).uniform(-14, 8.8, 2000)])
    got = kv8.round_e4m3(x)
    for a, b in zip(x, got):  # nearest; of two equally near, the even code
        d = np.abs(v - a)
        near = np.flatnonzero(d == d.min())
        want = near[0] if len(near) == 1 else [i for i in near if i % 2 == 0][0]
        assert b == v[want], a
    assert np.array_equal(kv8.round_e4m3(-x), -got)
    t = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, kv8.round_e4m3(x.astype(np.float32)))


def test_oracle_exponent():
    for amax, e in ((0.0, -100), (448.0, 0), (448.0001, 1), (224.0, -1), (1.0, -8), (1.75, -8),
                    (1.7501, -7), (2.0 ** -90, -98), (2.0 ** -120, -100), (3.3e38, 120)):
        assert kv8.exponent(amax) == e, amax


@pytest.mark.parametrize("chunks", [[16], [1] * 16, [3, 5, 8], [7, 9], [15, 1]])
def test_oracle_append_keeps_values_close(chunks):
    """Whatever the appends to a block, a value is off by at most half a step of
    its own (2^-4 of it) or of the smallest code, once for each rounding: the
    first one and one for each growth of the scale, which only adds the latter."""
    r = np.random.default_rng(len(chunks))
    k = r.standard_normal((16, 2, 64)) * np.exp(r.standard_normal((16, 1, 1)))
    kc, vc = np.zeros((3, 2, 16, 64)), np.zeros((3, 2, 64, 16))
    ex = kv8.new_exponents(3, 2)
    a = 0
    for n in chunks:
        kv8.append(kc, vc, ex, [[1]], [a + n], [0, n], k[a:a + n], -k[a:a + n])
        a += n
    assert np.array_equal(kc[1].transpose(0, 2, 1), -vc[1])
    for h in range(2):
        step = 2.0 ** (ex[1, h, 0] - 9)
        err = np.abs(kc[1, h] - k[:, h])
        assert np.all(err <= 2.0 ** -4 * np.abs(k[:, h]) + len(chunks) * step / 2)
        assert np.abs(k[:, h]).max() <= 448 * 2.0 ** ex[1, h, 0]
    assert not kc[0].any() and not kc[2].any()


def shape(seqs, head_dim=128, dtype=None):
    lens = np.array([x for x, _ in seqs], np.int32)
    cu = np.concatenate([[0], np.cumsum([q for _, q in seqs])]).astype(np.int32)
    return lens, cu


@pytest.mark.parametrize("seqs,kind,n_q", [([(2300, 1)] * 5, B.KIND_DECODE, 1),
                                           ([(700, 5)] * 3, B.KIND_VERIFY, 5),
                                           ([(900, 300), (17, 17), (40, 0)], B.KIND_PREFILL, 0)])
def test_plans(seqs, kind, n_q):
    lens, cu = shape(seqs)
    plan, info = B.plan(kind, n_q, lens, cu, 8, 2, 128, 16, B.PA_BF16_KV8)
    assert info.dtype == B.PA_BF16_KV8 and info.grid > 0 and info.plan_words == plan.size
    assert info.workspace_bytes <= B.workspace_size(int(cu[-1]), 8, 128, int(lens.max()))
    with pytest.raises(B.PaError) as e:
        B.plan(kind, n_q, lens, cu, 8, 2, 128, 16, 3)
    assert e.value.code == "unsupported"


def rows_args(**kw):
    """Valid arguments of pa_kv8_append / pa_kv8_read, changed by name."""
    a = dict(k=256, ks=256, v=512, vs=256, bt=64, mb=4, sl=64, cu=64, n_seqs=2, n=5, kc=1024,
             vc=2048, sc=64, nb=16, hkv=2, d=128, bs=16, dtype=B.PA_BF16, stream=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("name", ["pa_kv8_append", "pa_kv8_read"])
def test_rows_refusals(name):
    fn = getattr(B.lib(), name)
    for kw, code in (({"d": 96}, B.PA_ERR_UNSUPPORTED), ({"bs": 32}, B.PA_ERR_UNSUPPORTED),
                     ({"dtype": 2}, B.PA_ERR_UNSUPPORTED), ({"dtype": 7}, B.PA_ERR_UNSUPPORTED),
                     ({"nb": 0}, B.PA_ERR_ARG), ({"hkv": 0}, B.PA_ERR_ARG),
                     ({"nb": 1 << 28}, B.PA_ERR_ARG), ({"n": -1}, B.PA_ERR_ARG),
                     ({"n_seqs": -1}, B.PA_ERR_ARG), ({"mb": 0}, B.PA_ERR_ARG),
                     ({"ks": 255}, B.PA_ERR_ARG), ({"vs": 128}, B.PA_ERR_ARG),
                     ({"ks": 260}, B.PA_ERR_ARG), ({"k": 264}, B.PA_ERR_ARG),
                     ({"v": 520}, B.PA_ERR_ARG), ({"kc": 1032}, B.PA_ERR_ARG),
                     ({"vc": 2052}, B.PA_ERR_ARG), ({"sc": 66}, B.PA_ERR_ARG)):
        assert fn(*rows_args(**kw)) == code, kw
        assert name.encode() in B.lib().pa_last_error()
    for p in ("k", "v", "bt", "sl", "cu", "kc", "vc", "sc"):
        assert fn(*rows_args(**{p: None})) == B.PA_ERR_ARG, p
        assert b"NULL" in B.lib().pa_last_error()
    # nothing to do: no pointer is looked at
    none = dict(k=None, v=None, bt=None, sl=None, cu=None, kc=None, vc=None, sc=None)
    assert fn(*rows_args(n=0, **none)) == B.PA_OK
    assert fn(*rows_args(n_seqs=0, **none)) == B.PA_OK


def test_attention_refusals():
    lib = B.lib()
    info = B.PlanInfo()
    info.kind = B.KIND_DECODE
    info.n_seqs, info.total_q, info.num_q_heads, info.num_kv_heads = 1, 1, 8, 2
    info.head_dim, info.dtype, info.variant = 128, B.PA_BF16_KV8, 1
    names = ["q", "kc", "vc", "sc", "nb", "bt", "mb", "sl", "cu", "n", "T", "hq", "hkv", "d", "bs",
             "scale", "plan", "info", "ws", "wsb", "out", "lse", "stream"]
    good = dict(q=256, kc=1024, vc=2048, sc=64, nb=16, bt=64, mb=4, sl=64, cu=64, n=1, T=1, hq=8,
                hkv=2, d=128, bs=16, scale=0.1, plan=64, info=ctypes.byref(info), ws=None, wsb=0,
                out=512, lse=None, stream=None)

    def call(fn, **kw):
        a = dict(good, **kw)
        drop = ("ws", "wsb") if "noalloc" in fn else ()
        return getattr(lib, fn)(*[a[n] for n in names if n not in drop])

    for fn in ("pa_kv8_attn_decode", "pa_kv8_attn_decode_noalloc"):
        for kw, code in (({"d": 96}, B.PA_ERR_UNSUPPORTED), ({"bs": 32}, B.PA_ERR_UNSUPPORTED),
                         ({"hq": 7}, B.PA_ERR_ARG), ({"scale": 0.0}, B.PA_ERR_ARG),
                         ({"scale": float("inf")}, B.PA_ERR_ARG), ({"nb": 0}, B.PA_ERR_ARG),
                         ({"info": None}, B.PA_ERR_ARG), ({"mb": 0}, B.PA_ERR_ARG),
                         ({"q": 264}, B.PA_ERR_ARG), ({"kc": 1028}, B.PA_ERR_ARG),
                         ({"vc": 2056}, B.PA_ERR_ARG), ({"out": 514}, B.PA_ERR_ARG),
                         ({"sc": 66}, B.PA_ERR_ARG)):
            assert call(fn, **kw) == code, (fn, kw)
        for p in ("q", "kc", "vc", "sc", "bt", "sl", "cu", "plan", "out"):
            assert call(fn, **{p: None}) == B.PA_ERR_ARG, p
            assert b"NULL" in lib.pa_last_error()
    # another kind's plan, another launch's, and one for a bf16 cache
    assert call("pa_kv8_attn_prefill") == B.PA_ERR_ARG
    assert call("pa_kv8_attn_verify") == B.PA_ERR_ARG
    for field, val in (("n_seqs", 2), ("total_q", 3), ("num_q_heads", 16), ("num_kv_heads", 1),
                       ("head_dim", 64), ("dtype", B.PA_BF16)):
        bad = B.PlanInfo()
        ctypes.memmove(ctypes.byref(bad), ctypes.byref(info), ctypes.sizeof(info))
        setattr(bad, field, val)
        assert call("pa_kv8_attn_decode", info=ctypes.byref(bad)) == B.PA_ERR_ARG, field
        assert b"plan was built for" in lib.pa_last_error(), field
    # and a plan for the 8-bit cache is refused by the calls over a bf16 cache
    args = [256, 1024, 2048, 16, 64, 4, 64, 64, 1, 1, 8, 2, 128, 16, 0.1, B.PA_BF16, 64,
            ctypes.byref(info), None, 0, 512, None, None]
    assert lib.pa_attn_decode(*args) == B.PA_ERR_ARG
    args[15] = B.PA_BF16_KV8
    assert lib.pa_attn_decode(*args) == B.PA_ERR_UNSUPPORTED
    assert lib.pa_kv_append(256, 512, 64, 3, 1024, 2048, 16, 2, 128, 16, B.PA_BF16_KV8,
                            None) == B.PA_ERR_UNSUPPORTED
    # a workspace smaller than the plan's
    info.partial_rows = 4
    info.workspace_bytes = 4 * 129 * 4
    assert call("pa_kv8_attn_decode") == B.PA_ERR_ARG
    assert b"workspace" in lib.pa_last_error()
    info.partial_rows = 70000
    info.workspace_bytes = 70000 * 129 * 4
    assert call("pa_kv8_attn_decode_noalloc") == B.PA_ERR_ARG
    assert b"workspace" in lib.pa_last_error()


def test_norm_rope_refusals():
    fn = B.lib().pa_qk_norm_rope
    good = dict(q=256, qs=1024, k=512, ks=256, pos=64, n=3, table=64, n_pos=8, rot=128, qw=128,
                kw=128, eps=1e-6, flags=1, qo=1024, ko=2048, hq=8, hkv=2, d=128, dtype=B.PA_BF16,
                stream=None)
    for kw, code in (({"d": 96}, B.PA_ERR_UNSUPPORTED), ({"dtype": 2}, B.PA_ERR_UNSUPPORTED),
                     ({"hq": -1}, B.PA_ERR_ARG), ({"hq": 0, "hkv": 0}, B.PA_ERR_ARG),
                     ({"n": -1}, B.PA_ERR_ARG), ({"n_pos": -1}, B.PA_ERR_ARG),
                     ({"rot": 130}, B.PA_ERR_ARG), ({"rot": 7}, B.PA_ERR_ARG),
                     ({"rot": -2}, B.PA_ERR_ARG), ({"flags": 4}, B.PA_ERR_ARG),
                     ({"eps": -1.0}, B.PA_ERR_ARG), ({"eps": float("nan")}, B.PA_ERR_ARG),
                     ({"qs": 1016}, B.PA_ERR_ARG), ({"ks": 255}, B.PA_ERR_ARG),
                     ({"qs": 1028}, B.PA_ERR_ARG), ({"q": 264}, B.PA_ERR_ARG),
                     ({"ko": 2050}, B.PA_ERR_ARG), ({"qw": 136}, B.PA_ERR_ARG),
                     ({"table": 66}, B.PA_ERR_ARG)):
        assert fn(*dict(good, **kw).values()) == code, kw
        assert b"pa_qk_norm_rope" in B.lib().pa_last_error()
    for p in ("q", "k", "pos", "table", "qo", "ko"):
        assert fn(*dict(good, **{p: None}).values()) == B.PA_ERR_ARG, p
        assert b"NULL" in B.lib().pa_last_error()
    assert fn(*dict(good, n=0, q=None, pos=None).values()) == B.PA_OK


def test_binding_refusals():
    """Tensors whose types, shapes or strides the calls do not take."""
    nb, hkv, d = 4, 2, 128
    sk, sv, ss = B.kv8_cache_shapes(nb, hkv, d)
    k, v = (torch.zeros(s, dtype=torch.uint8).view(torch.float8_e4m3fn) for s in (sk, sv))
    sc = torch.zeros(ss, dtype=torch.uint8)
    bt = torch.zeros((1, 2), dtype=torch.int32)
    sl, cu = torch.tensor([3], dtype=torch.int32), torch.tensor([0, 3], dtype=torch.int32)
    rows = torch.zeros((3, hkv, d), dtype=torch.bfloat16)

    def bad(code, fn, *a, **kw):
        with pytest.raises(B.PaError) as e:
            fn(*a, **kw)
        assert e.value.code == code, e.value

    meta = (bt, sl, cu)
    for fn in (B.kv8_append, B.kv8_read):
        bad("unsupported", fn, rows, rows, *meta, k.view(torch.int8), v, sc)
        bad("arg", fn, rows, rows, *meta, k, v, sc[:3])
        bad("arg", fn, rows, rows, *meta, v, v, sc)
        bad("arg", fn, rows, rows[:2], *meta, k, v, sc)
        bad("arg", fn, rows, rows.float(), *meta, k, v, sc)
        bad("arg", fn, rows[:, :1], rows[:, :1], *meta, k, v, sc)
        bad("arg", fn, rows.transpose(1, 2).contiguous().transpose(1, 2), rows, *meta, k, v, sc)
        bad("arg", fn, rows, rows, bt, sl.long(), cu, k, v, sc)
        bad("arg", fn, rows, rows, bt, sl, cu[:1], k, v, sc)
        bad("unsupported", fn, rows.half(), rows.half(), *meta, k, v, sc)
    q = torch.zeros((3, 8, d), dtype=torch.bfloat16)
    info = B.PlanInfo()
    for kw, code in ((dict(q=q.float()), "unsupported"), (dict(out=q[:2]), "arg"),
                     (dict(q=q[..., :64]), "arg"), (dict(lse=torch.zeros(3, 8).double()), "arg"),
                     (dict(lse=torch.zeros(3, 4)), "arg")):
        a = dict(q=q, out=q, lse=None)
        a.update(kw)
        bad(code, B.kv8_attention, B.KIND_PREFILL, a["q"], k, v, sc, *meta, bt, info, None,
            a["out"], a["lse"])
    # a plan shorter than its info says, one of another type
    info.plan_words = 100
    for plan in (torch.zeros(99, dtype=torch.int32), torch.zeros(200, dtype=torch.int64)):
        bad("arg", B.kv8_attention, B.KIND_PREFILL, q, k, v, sc, *meta, plan, info, None, q)
    # everything in order but for the device: a host tensor is refused
    info.plan_words = 1
    for call in (lambda: B.kv8_append(rows, rows, *meta, k, v, sc),
                 lambda: B.kv8_attention(B.KIND_PREFILL, q, k, v, sc, *meta, bt, info, None, q),
                 lambda: B.kv8_attention_decode_noalloc(q, k, v, sc, *meta, bt, info, q),
                 lambda: B.qk_norm_rope(q, rows, torch.zeros(3, dtype=torch.int32),
                                        torch.zeros((8, d)), q, rows)):
        with pytest.raises(B.PaError) as e:
            call()
        assert e.value.code == "arg" and "GPU" in str(e.value)
    pos, tab = torch.zeros(3, dtype=torch.int32), torch.zeros((8, d))
    bad("arg", B.qk_norm_rope, q, rows[:2], pos, tab, q, rows)
    bad("arg", B.qk_norm_rope, q, rows, pos.long(), tab, q, rows)
    bad("arg", B.qk_norm_rope, q, rows, pos[:2], tab, q, rows)
    bad("arg", B.qk_norm_rope, q, rows, pos, tab.double(), q, rows)
    bad("arg", B.qk_norm_rope, q, rows, pos, tab, q[:2], rows)
    bad("arg", B.qk_norm_rope, q, rows, pos, tab, q, rows.float())
    bad("arg", B.qk_norm_rope, q, rows, pos, tab, q, rows, q_weight=torch.zeros(d))
    bad("arg", B.qk_norm_rope, q, rows.float(), pos, tab, q, rows)


def check_plan8(plan, info, L, q, G, hkv, D):
    """Every (sequence, kv-head, row) is produced exactly once, by one item or by
    parts whose key ranges tile its keys and whose partial rows are its merge
    group's; the four items of a joined workgroup hold the same rows over adjacent
    keys, at most 64 blocks each, and count as one."""
    from tests.test_capi_host import parse_plan
    h, shared, tiles, rows, groups = parse_plan(plan)
    assert h[0] == 0x31304150 and len(rows) % 4 == 0
    assert info.grid == len(shared) + h[3] + len(rows) // 4
    assert bool(info.variant & 2) == any(t[3] > 16 for t in rows if t[0] >= 0)
    items = list(tiles)
    for i in range(0, len(rows), 4):
        quad = rows[i:i + 4]
        assert all(t[5] - t[4] <= 1024 and t[3] <= 32 for t in quad if t[0] >= 0)
        if quad[0][7] & 2:
            assert all(t[:4] + t[6:] == quad[0][:4] + quad[0][6:] and t[0] >= 0 for t in quad)
            assert all(a[5] == b[4] and b[4] <= b[5] for a, b in zip(quad, quad[1:]))
            assert quad[0][4] < quad[0][5] <= quad[3][5] and quad[0][4] % 16 == 0
            assert all(t[4] % 16 == 0 for t in quad if t[4] < t[5])
            items.append(quad[0][:5] + [quad[3][5]] + quad[0][6:])
        else:
            items += [t for t in quad if t[0] >= 0]
            assert not any(t[7] & 2 for t in quad)
        # items of sequences with more rows than one holds say so
        assert all(bool(t[7] & 4) == (q[t[0]] * G > 32) for t in quad if t[0] >= 0)
    cover, writes = {}, []
    for seq, kvh, row0, nrows, kv0, kv1, part, _ in items:
        assert kv0 % 16 == 0 and 0 <= kv0 < kv1 <= L[seq]
        for lr in range(nrows):
            cover.setdefault((seq, kvh, row0 + lr), []).append((kv0, kv1, part + lr if part >= 0 else -1))
    for moff, kvh, row0, nrows, kv0, kv1, rpm, bseq, poff in shared:
        assert kv0 % 64 == 0 and kv1 % 64 == 0
        for rg in range(row0, row0 + nrows):
            m, rl = divmod(rg, rpm)
            seq, base = plan[moff + 2 * m], plan[moff + 2 * m + 1] + poff
            assert kv1 <= L[seq] - q[seq]
            cover.setdefault((seq, kvh, rl), []).append((kv0, kv1, base + rl))
    expected = {}
    for seq, kvh, row0, nrows, nsplit, part, stride, _ in groups:
        for lr in range(nrows):
            expected[(seq, kvh, row0 + lr)] = {part + sp * stride + lr for sp in range(nsplit)}
    assert len(cover) == int(q.sum()) * G * hkv
    for (seq, kvh, rho), ranges in cover.items():
        ranges.sort()
        if len(ranges) == 1 and ranges[0][2] < 0:
            assert (seq, kvh, rho) not in expected and ranges[0][0] == 0
            assert ranges[0][1] >= L[seq] - q[seq] + rho // G + 1
        else:
            parts = [p for _, _, p in ranges]
            assert set(parts) == expected[(seq, kvh, rho)] and len(set(parts)) == len(parts)
            assert ranges[0][0] == 0 and ranges[-1][1] == L[seq]
            assert all(a[1] == b[0] for a, b in zip(ranges, ranges[1:]))
            writes += parts
    assert sorted(writes) == list(range(int(info.partial_rows)))
    assert int(info.workspace_bytes) == int(info.partial_rows) * (D + 1) * 4
    assert B.workspace_size(int(q.sum()), hkv * G, D, int(max(L))) >= int(info.workspace_bytes)
    return tiles, rows


@pytest.mark.parametrize("seed", range(30))
def test_plans_cover_every_row_once(seed):
    """Random launches over the 8-bit cache, prefixes shared, rows of every item
    kind (sequences of 33 to 64 rows run as two row items)."""
    r = np.random.default_rng(seed)
    n, hkv, G = int(r.integers(1, 40)), int(r.choice([1, 2, 8])), int(r.choice([1, 4, 7, 8, 40, 64]))
    L = r.integers(1, 4000, size=n)
    q = np.minimum(L, r.choice([1, 2, 5, 8, 9, 33, 300], size=n))
    kind, n_q = B.KIND_PREFILL, 0
    if seed % 3:
        n_q = 1 if seed % 3 == 1 else 5
        L = np.maximum(L, n_q)
        q[:] = n_q
        kind = B.KIND_DECODE if n_q == 1 else B.KIND_VERIFY
    cu = np.concatenate([[0], np.cumsum(q)])
    mb = int((L.max() + 15) // 16)
    bt = np.full((n, mb), -1, np.int32)
    nxt, prefix = 0, int(r.integers(0, 200))
    for s in range(n):
        nb = int((L[s] + 15) // 16)
        pb = min(nb - 1, prefix) if r.random() < 0.6 else 0
        bt[s, :pb] = 10 ** 6 + np.arange(pb)
        bt[s, pb:nb] = nxt + np.arange(nb - pb)
        nxt += nb - pb
    D = int(r.choice([64, 128]))
    plan, info = B.plan(kind, n_q, L, cu, hkv * G, hkv, D, 16, B.PA_BF16_KV8, block_table=bt)
    tiles, rows = check_plan8(plan, info, L, q, G, hkv, D)
    cfg = synth.AttnConfig("", "bf16", hkv * G, hkv, D, 16, 0)
    assert info.plan_words <= plan_words_bound(cfg, n, int(cu[-1]), mb)
    assert all(q[t[0]] * G <= 64 for t in rows if t[0] >= 0)
    if kind != B.KIND_DECODE:
        assert all(q[t[0]] * G > 64 for t in tiles)
    else:  # tiles only where the array of the call without workspace asks for them
        assert info.workspace_bytes <= B.NOALLOC_WORKSPACE_BYTES


@pytest.mark.parametrize("seed", range(12))
def test_plan_bound_without_the_8_bit_cache(seed):
    """Callers that plan for bf16 and float32 caches only need not hold its row items."""
    r = np.random.default_rng([seed, 3])
    n, hkv, G = int(r.integers(1, 60)), int(r.choice([1, 2, 8])), int(r.choice([1, 4, 8, 40]))
    L = r.integers(1, 5000, size=n)
    q = np.minimum(L, r.choice([1, 2, 5, 33, 300], size=n))
    kind = B.KIND_PREFILL
    if seed % 2:
        q[:], kind = 1, B.KIND_DECODE
    cu = np.concatenate([[0], np.cumsum(q)])
    mb = int((L.max() + 15) // 16)
    cfg = synth.AttnConfig("", "bf16", hkv * G, hkv, 128, 16, 0)
    least = plan_words_bound(cfg, n, int(cu[-1]), mb, kv8=False)
    # tiles, key-split items and merge groups, 8 words each, and what does not grow
    assert least == 16416 + 8 * (hkv * (int(cu[-1]) * G // 128 + n)
                                 + 2 * hkv * n * (mb * 16 // 256 + 2) + 64)
    assert least < plan_words_bound(cfg, n, int(cu[-1]), mb)
    for dtype in (B.PA_BF16, B.PA_F32):
        _, info = B.plan(kind, 1, L, cu, hkv * G, hkv, 128, 16, dtype)
        assert info.plan_words <= least


@pytest.mark.parametrize("q", [1, 5])
@pytest.mark.parametrize("num_cus, shared", [(256, False), (23, False), (22, True)])
def test_small_launches_leave_shared_prefixes_to_their_row_items(q, num_cus, shared):
    """Up to 768 keys per CU: 4 sequences of 8580 keys together are 17160 for 2 kv-heads."""
    L = np.array([2100, 2130, 2160, 2190])
    bt = np.full((4, 137), -1, np.int32)
    for s in range(4):
        bt[s, :128] = np.arange(128)
        bt[s, 128:] = 128 + 9 * s + np.arange(9)
    kind = B.KIND_DECODE if q == 1 else B.KIND_VERIFY
    plan, info = B.plan(kind, q, L, np.arange(5) * q, 16, 2, 128, 16, B.PA_BF16_KV8,
                        num_cus=num_cus, block_table=bt)
    assert (info.n_shared_items > 0) == shared
    check_plan8(plan, info, L, np.full(4, q), 8, 2, 128)
    # beside a prefill chunk they are split off
    n = np.array([q, q, q, 300])
    plan, info = B.plan(B.KIND_PREFILL, 0, L, np.concatenate([[0], np.cumsum(n)]), 16, 2, 128, 16,
                        B.PA_BF16_KV8, num_cus=num_cus, block_table=bt)
    assert info.n_shared_items > 0
    check_plan8(plan, info, L, n, 8, 2, 128)


@pytest.mark.parametrize("d, q, num_cus, shared", [(64, 5, 256, True), (64, 5, 304, False),
                                                   (64, 1, 256, False), (128, 5, 256, False)])
def test_small_verifications_split_shared_prefixes_off(d, q, num_cus, shared):
    """At head_dim 64, where their row workgroups (joined fours of up to 384 keys each) are
    more than the CUs: 8 sequences of 3000 keys and 8 kv-heads come to more than 256."""
    L = np.array([2848 + 40 * i for i in range(8)])
    bt = np.full((8, 200), -1, np.int32)
    for s in range(8):
        bt[s, :128] = np.arange(128)
        n = (int(L[s]) + 15) // 16 - 128
        bt[s, 128:128 + n] = 128 + 80 * s + np.arange(n)
    kind = B.KIND_DECODE if q == 1 else B.KIND_VERIFY
    plan, info = B.plan(kind, q, L, np.arange(9) * q, 32, 8, d, 16, B.PA_BF16_KV8,
                        num_cus=num_cus, block_table=bt)
    assert (info.n_shared_items > 0) == shared
    check_plan8(plan, info, L, np.full(8, q), 4, 8, d)
