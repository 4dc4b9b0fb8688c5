"""The 4-bit cache, attention weights and eviction on the host: the oracle's rounding
against brute force, plans, the pool's side of an eviction against its oracle, and every
refusal of the entry points (made before anything is launched: the pointers below are never
read)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import apc, kv4
from paper_2605_11232_amd import binding as B
from paper_2605_11232_amd.runtime import plan_words_bound
from tests.test_kv8_host import check_plan8, rows_args, shape


# ---- the oracle -------------------------------------------------------------------------------

def test_oracle_codes_are_nearest_even():
    v = kv4.NUMBERS
    mid = (v[1:] + v[:-1]) / 2
    x = np.concatenate([v, mid, np.nextafter(mid, 0), np.nextafter(mid, 9), [6.5, 7.0, 100.0],
                        np.random.default_rng(1).uniform(0, 7, 3000)])
    for a, c in zip(x, kv4.codes(x)):
        d = np.abs(v - a)
        near = np.flatnonzero(d == d.min())
        assert c == (near[0] if len(near) == 1 else [i for i in near if i % 2 == 0][0]), a
    assert np.array_equal(kv4.codes(-x), kv4.codes(x) + 8)
    assert np.array_equal(kv4.values(np.arange(16)[None], np.array([128]))[0], 2 * np.concatenate([v, -v]))


def test_oracle_exponents():
    for amax, e in ((0.0, -100), (7.0, 0), (7.001, 1), (3.5, -1), (1.0, -2), (1.75, -2), (1.76, -1),
                    (2.0 ** -120, -100), (3.3e38, 100), (np.inf, 101), (np.nan, 101)):
        assert kv4.exponents(np.array([0.0, -amax])) == e, amax
    r = np.random.default_rng(2)
    x = r.standard_normal((200, 32)) * np.exp(5 * r.standard_normal((200, 1)))
    y = kv4.values(*kv4.quantise(x))
    top = np.abs(x).max(1, keepdims=True)
    # half a step of the code: a quarter of the value, or of the smallest code's scale
    assert np.all(np.abs(x - y) <= np.maximum(np.abs(x) / 4, np.exp2(kv4.exponents(x))[:, None] / 4))
    assert np.all(np.exp2(kv4.exponents(x))[:, None] * 7 >= top)


# ---- plans ------------------------------------------------------------------------------------

@pytest.mark.parametrize("seqs,kind,n_q", [([(2300, 1)] * 5, B.KIND_DECODE, 1),
                                           ([(700, 5)] * 3, B.KIND_VERIFY, 5),
                                           ([(900, 300), (17, 17), (40, 0)], B.KIND_PREFILL, 0)])
def test_plans(seqs, kind, n_q):
    lens, cu = shape(seqs)
    plan, info = B.plan(kind, n_q, lens, cu, 8, 2, 128, 16, B.PA_BF16_KV4)
    assert info.dtype == B.PA_BF16_KV4 and info.grid > 0 and info.plan_words == plan.size
    assert info.workspace_bytes <= B.workspace_size(int(cu[-1]), 8, 128, int(lens.max()))


@pytest.mark.parametrize("seed", range(20))
def test_plans_cover_every_row_once(seed):
    """Random launches, prefixes shared, rows of every item kind, within the plan bound."""
    r = np.random.default_rng([seed, 4])
    n, hkv, G = int(r.integers(1, 40)), int(r.choice([1, 2, 8])), int(r.choice([1, 4, 7, 8, 40, 64]))
    L = r.integers(1, 4000, size=n)
    q = np.minimum(L, r.choice([1, 2, 5, 8, 9, 33, 300], size=n))
    kind, n_q = B.KIND_PREFILL, 0
    if seed % 3:
        kind, n_q = (B.KIND_DECODE, 1) if seed % 3 == 1 else (B.KIND_VERIFY, int(r.integers(1, 9)))
        L = np.maximum(L, n_q)
        q = np.full(n, n_q)
    d = int(r.choice([64, 128]))
    width = int(max(-(-L // 16)))
    table = np.arange(n * width, dtype=np.int32).reshape(n, width)
    shared = int(r.integers(0, 60))
    table[:, :shared] = table[0, :shared]
    cu = np.concatenate([[0], np.cumsum(q)]).astype(np.int32)
    plan, info = B.plan(kind, n_q, L.astype(np.int32), cu, hkv * G, hkv, d, 16, B.PA_BF16_KV4,
                        block_table=table)
    check_plan8(plan, info, L, q, G, hkv, d)

    class cfg:
        block_size, group, num_kv_heads = 16, G, hkv
    assert info.plan_words <= plan_words_bound(cfg, n, int(q.sum()), width)


# ---- the pool ---------------------------------------------------------------------------------

CODES = {"arg": apc.ArgError, "no_blocks": apc.NoBlocksError, "unknown_seq": apc.UnknownSeqError}


@pytest.mark.parametrize("evict", [False, True])
@pytest.mark.parametrize("seed", range(6))
def test_compaction_against_the_oracle(seed, evict):
    """Random admissions, extensions, truncations, compactions and releases: the same
    blocks, free lists, counters and refusals."""
    r = np.random.default_rng([seed, 7])
    order = r.permutation(60).astype(np.int32)
    pool, orc = B.Pool(60, 4, order, evict=evict), apc.PrefixCacheOracle(60, 4, order)
    orc.evict = evict
    prefixes = [list(r.integers(0, 9, 24)) for _ in range(3)]
    live, next_id, refused = [], 0, 0
    for _ in range(400):
        op = r.choice(["add", "extend", "truncate", "compact", "compact", "free"])
        sid = int(r.choice(live)) if live and r.random() < 0.97 else next_id
        if op == "add":
            sid = next_id
            next_id += 1
            args = [prefixes[r.integers(3)][:r.integers(1, 25)] + list(r.integers(0, 9, r.integers(0, 12)))]
        elif op == "extend":
            args = [list(r.integers(0, 9, r.integers(0, 10)))]
        elif op == "truncate":
            args = [int(r.integers(0, 40))]
        elif op == "compact":
            n = int(r.integers(0, 40))
            args = [n, int(r.integers(-1, n + 2)), bool(r.integers(2))]
        else:
            args = []
        want = None
        try:
            getattr(orc, {"free": "free_seq"}.get(op, op))(sid, *args)
        except apc.OracleError as e:
            want = type(e)
        try:
            getattr(pool, op)(sid, *args)
            assert want is None, (op, args)
        except B.PaError as e:
            refused += 1
            assert want is CODES[e.code], (op, args, e)
        if want is None and op in ("add", "free"):
            live = live + [sid] if op == "add" else [x for x in live if x != sid]
        assert pool.free_list() == orc.free_list() and pool.stats() == orc.stats()
        for x in live:
            assert pool.blocks_of(x) == orc.blocks_of(x) and pool.seq_len(x) == orc.seq_len(x)
    assert refused > 5
    for x in live:
        pool.free(x), orc.free_seq(x)
    assert pool.free_list() == orc.free_list() and pool.stats() == orc.stats()


def test_compacted_blocks_are_not_a_prefix():
    """What a shortened sequence holds is never offered to another request; the blocks that
    it gave back cached still are."""
    pool = B.Pool(40, 16, np.arange(40, dtype=np.int32))
    toks = list(range(100))
    pool.add(1, toks[:40])
    pool.extend(1, toks[40:])
    pool.compact(1, 50, 32, in_place=True)
    assert pool.seq_len(1) == 50 and len(pool.blocks_of(1)) == 4
    pool.extend(1, list(range(200, 230)))
    pool.free(1)
    assert pool.add(2, toks) == 32  # the prompt's full blocks, nothing behind them
    old = pool.blocks_of(2)
    pool.compact(2, 30, 0)
    assert not set(old) & set(pool.blocks_of(2)) and len(pool.blocks_of(2)) == 2
    assert pool.add(3, toks) == 96 and pool.blocks_of(3)[:6] == old[:6]
    with pytest.raises(B.PaError) as e:
        pool.compact(3, 90, 40, in_place=True)  # blocks of its cached prompt would change
    assert e.value.code == "arg"


# ---- refusals ---------------------------------------------------------------------------------

@pytest.mark.parametrize("name", ["pa_kv4_append", "pa_kv4_read"])
def test_rows_refusals(name):
    fn = getattr(B.lib(), name)
    for kw, code in (({"d": 96}, B.PA_ERR_UNSUPPORTED), ({"bs": 32}, B.PA_ERR_UNSUPPORTED),
                     ({"dtype": 2}, B.PA_ERR_UNSUPPORTED), ({"dtype": 4}, B.PA_ERR_UNSUPPORTED),
                     ({"nb": 0}, B.PA_ERR_ARG), ({"hkv": 0}, B.PA_ERR_ARG),
                     ({"nb": 1 << 28}, B.PA_ERR_ARG), ({"n": -1}, B.PA_ERR_ARG),
                     ({"n_seqs": -1}, B.PA_ERR_ARG), ({"mb": 0}, B.PA_ERR_ARG),
                     ({"ks": 255}, B.PA_ERR_ARG), ({"vs": 128}, B.PA_ERR_ARG),
                     ({"ks": 260}, B.PA_ERR_ARG), ({"k": 264}, B.PA_ERR_ARG),
                     ({"v": 520}, B.PA_ERR_ARG), ({"kc": 1032}, B.PA_ERR_ARG),
                     ({"vc": 2052}, B.PA_ERR_ARG), ({"sc": 72}, B.PA_ERR_ARG)):
        assert fn(*rows_args(**kw)) == code, kw
        assert name.encode() in B.lib().pa_last_error()
    for p in ("k", "v", "bt", "sl", "cu", "kc", "vc", "sc"):
        assert fn(*rows_args(**{p: None})) == B.PA_ERR_ARG, p
        assert b"NULL" in B.lib().pa_last_error()
    none = dict(k=None, v=None, bt=None, sl=None, cu=None, kc=None, vc=None, sc=None)
    assert fn(*rows_args(n=0, **none)) == B.PA_OK
    assert fn(*rows_args(n_seqs=0, **none)) == B.PA_OK


def test_attention_refusals():
    lib = B.lib()
    info = B.PlanInfo()
    info.kind = B.KIND_DECODE
    info.n_seqs, info.total_q, info.num_q_heads, info.num_kv_heads = 1, 1, 8, 2
    info.head_dim, info.dtype, info.variant = 128, B.PA_BF16_KV4, 1
    names = ["q", "kc", "vc", "sc", "nb", "bt", "mb", "sl", "cu", "n", "T", "hq", "hkv", "d", "bs",
             "scale", "plan", "info", "ws", "wsb", "out", "lse", "stream"]
    good = dict(q=256, kc=1024, vc=2048, sc=64, nb=16, bt=64, mb=4, sl=64, cu=64, n=1, T=1, hq=8,
                hkv=2, d=128, bs=16, scale=0.1, plan=64, info=ctypes.byref(info), ws=None, wsb=0,
                out=512, lse=None, stream=None)

    def call(fn, **kw):
        a = dict(good, **kw)
        drop = ("ws", "wsb") if "noalloc" in fn else ()
        return getattr(lib, fn)(*[a[n] for n in names if n not in drop])

    for fn in ("pa_kv4_attn_decode", "pa_kv4_attn_decode_noalloc"):
        for kw, code in (({"d": 96}, B.PA_ERR_UNSUPPORTED), ({"bs": 32}, B.PA_ERR_UNSUPPORTED),
                         ({"hq": 7}, B.PA_ERR_ARG), ({"scale": 0.0}, B.PA_ERR_ARG),
                         ({"info": None}, B.PA_ERR_ARG), ({"mb": 0}, B.PA_ERR_ARG),
                         ({"q": 264}, B.PA_ERR_ARG), ({"kc": 1028}, B.PA_ERR_ARG),
                         ({"vc": 2056}, B.PA_ERR_ARG), ({"out": 514}, B.PA_ERR_ARG),
                         ({"sc": 72}, B.PA_ERR_ARG)):
            assert call(fn, **kw) == code, (fn, kw)
        for p in ("q", "kc", "vc", "sc", "bt", "sl", "cu", "plan", "out"):
            assert call(fn, **{p: None}) == B.PA_ERR_ARG, p
            assert b"NULL" in lib.pa_last_error()
    assert call("pa_kv4_attn_prefill") == B.PA_ERR_ARG
    assert call("pa_kv4_attn_verify") == B.PA_ERR_ARG
    # a plan for another cache, and this one at the calls over the others
    for dtype in (B.PA_BF16, B.PA_BF16_KV8):
        bad = B.PlanInfo()
        ctypes.memmove(ctypes.byref(bad), ctypes.byref(info), ctypes.sizeof(info))
        bad.dtype = dtype
        assert call("pa_kv4_attn_decode", info=ctypes.byref(bad)) == B.PA_ERR_ARG
        assert b"plan was built for" in lib.pa_last_error()
    assert call("pa_kv8_attn_decode") == B.PA_ERR_ARG
    args = [256, 1024, 2048, 16, 64, 4, 64, 64, 1, 1, 8, 2, 128, 16, 0.1, B.PA_BF16, 64,
            ctypes.byref(info), None, 0, 512, None, None]
    assert lib.pa_attn_decode(*args) == B.PA_ERR_ARG
    args[15] = B.PA_BF16_KV4
    assert lib.pa_attn_decode(*args) == B.PA_ERR_UNSUPPORTED
    info.partial_rows, info.workspace_bytes = 70000, 70000 * 129 * 4
    assert call("pa_kv4_attn_decode_noalloc") == B.PA_ERR_ARG
    assert b"pa_kv4_attn_decode with" in lib.pa_last_error()


def test_weights_refusals():
    fn = B.lib().pa_attn_weights
    good = dict(q=256, lse=64, kc=1024, sc=None, nb=16, bt=64, mb=4, sl=64, cu=64, n=2, T=3, hq=8,
                hkv=2, d=128, bs=16, scale=0.1, dtype=B.PA_BF16, w=64, ws=100, acc=0, stream=None)
    for kw, code in (({"d": 96}, B.PA_ERR_UNSUPPORTED), ({"bs": 32}, B.PA_ERR_UNSUPPORTED),
                     ({"dtype": B.PA_F32}, B.PA_ERR_UNSUPPORTED), ({"dtype": 3}, B.PA_ERR_UNSUPPORTED),
                     ({"dtype": B.PA_BF16_KV8}, B.PA_ERR_UNSUPPORTED), ({"hq": 7}, B.PA_ERR_ARG),
                     ({"hq": 0}, B.PA_ERR_ARG), ({"nb": 0}, B.PA_ERR_ARG), ({"n": -1}, B.PA_ERR_ARG),
                     ({"T": -1}, B.PA_ERR_ARG), ({"T": 1 << 30}, B.PA_ERR_ARG), ({"mb": 0}, B.PA_ERR_ARG),
                     ({"ws": -1}, B.PA_ERR_ARG), ({"acc": 2}, B.PA_ERR_ARG), ({"scale": 0.0}, B.PA_ERR_ARG),
                     ({"scale": float("nan")}, B.PA_ERR_ARG), ({"q": 264}, B.PA_ERR_ARG),
                     ({"kc": 1028}, B.PA_ERR_ARG), ({"w": 66}, B.PA_ERR_ARG), ({"lse": 62}, B.PA_ERR_ARG)):
        assert fn(*dict(good, **kw).values()) == code, kw
        assert b"pa_attn_weights" in B.lib().pa_last_error()
    for p in ("q", "lse", "kc", "bt", "sl", "cu", "w"):
        assert fn(*dict(good, **{p: None}).values()) == B.PA_ERR_ARG, p
        assert b"NULL" in B.lib().pa_last_error()
    assert fn(*dict(good, dtype=B.PA_BF16_KV4).values()) == B.PA_ERR_ARG  # no scales
    none = dict(q=None, lse=None, kc=None, bt=None, sl=None, cu=None, w=None)
    for kw in ({"n": 0}, {"T": 0}, {"ws": 0}):
        assert fn(*dict(good, **none, **kw).values()) == B.PA_OK


def test_evict_refusals():
    fn = B.lib().pa_kv_evict
    good = dict(w=64, wo=64, ws=100, bt=64, mb=4, nt=128, nmb=3, sl=64, nl=64, first=None, window=2,
                n=2, kc=1024, vc=2048, sc=None, nb=16, hkv=2, d=128, bs=16, dtype=B.PA_BF16, kept=64,
                ks=40, stream=None)
    for kw, code in (({"d": 96}, B.PA_ERR_UNSUPPORTED), ({"bs": 32}, B.PA_ERR_UNSUPPORTED),
                     ({"dtype": B.PA_BF16_KV8}, B.PA_ERR_UNSUPPORTED), ({"dtype": 3}, B.PA_ERR_UNSUPPORTED),
                     ({"nb": 0}, B.PA_ERR_ARG), ({"hkv": 0}, B.PA_ERR_ARG), ({"n": -1}, B.PA_ERR_ARG),
                     ({"window": -1}, B.PA_ERR_ARG), ({"mb": 0}, B.PA_ERR_ARG), ({"nmb": 0}, B.PA_ERR_ARG),
                     ({"ws": -1}, B.PA_ERR_ARG), ({"ks": -1}, B.PA_ERR_ARG), ({"nt": 64}, B.PA_ERR_ARG),
                     ({"kc": 1032}, B.PA_ERR_ARG), ({"vc": 2050}, B.PA_ERR_ARG), ({"w": 66}, B.PA_ERR_ARG),
                     ({"wo": 65}, B.PA_ERR_ARG), ({"kept": 62}, B.PA_ERR_ARG)):
        assert fn(*dict(good, **kw).values()) == code, kw
        assert b"pa_kv_evict" in B.lib().pa_last_error()
    for p in ("w", "wo", "bt", "sl", "nl", "kc", "vc", "kept"):
        assert fn(*dict(good, **{p: None}).values()) == B.PA_ERR_ARG, p
        assert b"NULL" in B.lib().pa_last_error()
    assert fn(*dict(good, dtype=B.PA_BF16_KV4).values()) == B.PA_ERR_ARG  # no scales
    none = dict(w=None, wo=None, bt=None, nt=None, sl=None, nl=None, kc=None, vc=None, kept=None)
    for kw in ({"n": 0}, {"ws": 0}, {"ks": 0}):
        assert fn(*dict(good, **none, **kw).values()) == B.PA_OK


def test_evict_refuses_weights_that_overlap_in_part():
    """2 x 3 x 100 weights: 2400 bytes; an array that begins inside the other one."""
    fn = B.lib().pa_kv_evict
    for step in (4, 400, 2396, -4, -2396):
        assert fn(8192, 8192 + step, 100, 64, 4, 128, 3, 64, 64, None, 2, 2, 1024, 2048, None, 16, 3, 128,
                  16, B.PA_BF16, 64, 40, None) == B.PA_ERR_ARG, step
        assert b"overlap" in B.lib().pa_last_error()


def bad(code, fn, *a, **kw):
    with pytest.raises(B.PaError) as e:
        fn(*a, **kw)
    assert e.value.code == code, e.value
    return str(e.value)


def test_binding_refusals_of_the_4_bit_cache():
    """Tensors whose types, shapes or strides the calls do not take."""
    nb, hkv, d = 4, 2, 128
    k, v, sc = (torch.zeros(s, dtype=torch.uint8) for s in B.kv4_cache_shapes(nb, hkv, d))
    meta = (torch.zeros((1, 2), dtype=torch.int32), torch.tensor([3], dtype=torch.int32),
            torch.tensor([0, 3], dtype=torch.int32))
    rows = torch.zeros((3, hkv, d), dtype=torch.bfloat16)
    for fn in (B.kv4_append, B.kv4_read):
        bad("unsupported", fn, rows, rows, *meta, k.view(torch.int8), v, sc)
        bad("arg", fn, rows, rows, *meta, k, v, sc[:3])
        bad("arg", fn, rows, rows, *meta, k, v, sc[:, :, :4])
        bad("arg", fn, rows, rows, *meta, v, v, sc)
        bad("arg", fn, rows, rows, *meta, k, k, sc)
        bad("arg", fn, rows, rows[:2], *meta, k, v, sc)
        bad("arg", fn, rows, rows.float(), *meta, k, v, sc)
        bad("arg", fn, rows, rows, meta[0], meta[1].long(), meta[2], k, v, sc)
        bad("unsupported", fn, rows.half(), rows.half(), *meta, k, v, sc)
        assert "GPU" in bad("arg", fn, rows, rows, *meta, k, v, sc)
    q = torch.zeros((3, 8, d), dtype=torch.bfloat16)
    info = B.PlanInfo()
    info.plan_words = 1
    bad("unsupported", B.kv4_attention, B.KIND_PREFILL, q.float(), k, v, sc, *meta, meta[0], info, None, q)
    bad("arg", B.kv4_attention, B.KIND_PREFILL, q[..., :64], k, v, sc, *meta, meta[0], info, None, q)
    bad("arg", B.kv4_attention, B.KIND_PREFILL, q, k, v, sc[:, :1], *meta, meta[0], info, None, q)
    assert "GPU" in bad("arg", B.kv4_attention, B.KIND_PREFILL, q, k, v, sc, *meta, meta[0], info, None, q)
    assert "GPU" in bad("arg", B.kv4_attention_decode_noalloc, q, k, v, sc, *meta, meta[0], info, q)


def test_binding_refusals_of_weights_and_eviction():
    nb, hkv, d, n = 4, 2, 128, 1
    k4, v4, sc = (torch.zeros(s, dtype=torch.uint8) for s in B.kv4_cache_shapes(nb, hkv, d))
    k = torch.zeros((nb, hkv, d // 32, 16, 32), dtype=torch.bfloat16)
    v = torch.zeros((nb, hkv, d, 16), dtype=torch.bfloat16)
    bt, sl, cu = (torch.zeros((n, 2), dtype=torch.int32), torch.tensor([3], dtype=torch.int32),
                  torch.tensor([0, 3], dtype=torch.int32))
    q, lse = torch.zeros((3, 8, d), dtype=torch.bfloat16), torch.zeros((3, 8))
    w = torch.zeros((n, hkv, 20))
    A = B.attention_weights
    for code, change in (("unsupported", dict(q=q.float())), ("unsupported", dict(k=k.float())),
                         ("unsupported", dict(k=k4)), ("unsupported", dict(scales=sc)),
                         ("arg", dict(q=q[..., :64])), ("arg", dict(lse=lse[:2])),
                         ("arg", dict(lse=lse.double())), ("arg", dict(w=w[:, :1])),
                         ("arg", dict(w=w[:0])), ("arg", dict(w=w.double())), ("arg", dict(w=w[0])),
                         ("arg", dict(k=k4, scales=sc[:, :, :2])), ("arg", dict(sl=sl.long())),
                         ("arg", dict(bt=bt[:0])), ("arg", dict(cu=cu[:1]))):
        a = dict(q=q, lse=lse, k=k, bt=bt, sl=sl, cu=cu, w=w, scales=None)
        a.update(change)
        s = a.pop("scales")
        bad(code, A, *a.values(), scales=s)
    assert "GPU" in bad("arg", A, q, lse, k, bt, sl, cu, w)
    assert "GPU" in bad("arg", A, q, lse, k4, bt, sl, cu, w, scales=sc)
    kept, nl = torch.zeros((n, hkv, 9), dtype=torch.int32), torch.tensor([2], dtype=torch.int32)
    k8 = torch.zeros((nb, hkv, d // 64, 16, 64), dtype=torch.uint8).view(torch.float8_e4m3fn)
    for code, change in (("unsupported", dict(k=k8)), ("unsupported", dict(k=k4)),
                         ("unsupported", dict(scales=sc)), ("arg", dict(v=v.float())),
                         ("arg", dict(v=v[:, :, :64])), ("arg", dict(kept=kept.long())),
                         ("arg", dict(kept=kept[:, :1])), ("arg", dict(w=w.double())),
                         ("arg", dict(nl=nl.long())), ("arg", dict(sl=torch.zeros(2, dtype=torch.int32))),
                         ("arg", dict(bt=bt[0])), ("arg", dict(first=nl.long())),
                         ("arg", dict(new_table=bt.long())), ("arg", dict(weights_out=w[..., :5])),
                         ("arg", dict(k=k4, v=v4, scales=sc[:2]))):
        a = dict(w=w, bt=bt, sl=sl, nl=nl, k=k, v=v, kept=kept)
        kw = {x: y for x, y in change.items() if x not in a}
        a.update({x: y for x, y in change.items() if x in a})
        bad(code, B.kv_evict, *a.values(), **kw)
    assert "GPU" in bad("arg", B.kv_evict, w, bt, sl, nl, k, v, kept)
    assert "GPU" in bad("arg", B.kv_evict, w, bt, sl, nl, k4, v4, kept, scales=sc, new_table=bt, first=nl)


def test_replay_of_one_cache_only():
    from paper_2605_11232_amd import synth
    from paper_2605_11232_amd.runtime import DeviceReplay
    wl = synth.workload("decode", scale=0.02, steps=1)
    with pytest.raises(ValueError):
        DeviceReplay(wl, device="cpu", kv8=True, kv4=True)
