"""Performance cases of the operators that make a cached context smaller.

Five operators, as one layer of a serving step calls them:

* ``append``: the step's new keys and values quantised into the paged 4-bit
  cache, and read back as the values that the codes stand for.
* ``read``: tokens of the 4-bit cache read back as rows.
* ``attn``: attention over the 4-bit cache: prefill, decode, verification and
  the mixed launch.
* ``weights``: how much attention each cached key got from a launch's queries:
  for each sequence, kv-head and key the sum of its probabilities over the rows
  that see it.
* ``evict``: of each sequence and kv-head, the heaviest tokens, the leading and
  the latest ones stay; their keys, values and weights move together.

The 4-bit cache holds e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
negatives), two in a byte, the first in the low half: keys [NB, Hkv, 16, D / 2],
a token's dimensions side by side; values [NB, Hkv, D / 32, 16, 16], where byte
8 a + o / 2 of row i holds tokens o and o + 1 of dimension 32 c + 16 a + i.
Scales [NB, Hkv, D / 32 + 1, 16] are powers of two 2^e as bytes e + 127: for each
token one for 32 dimensions of its key, and one for its value.  e is the smallest
of -100 .. 100 with amax <= 7 2^e (7 is where rounding ends at 6); codes are
rounded to nearest even.  What holds anything not finite has the byte 255 and
codes of zero, and stands for NaN.

The bf16 cache: keys [NB, Hkv, D / 32, 16, 32], a token at its offset with bits
2 and 3 exchanged; values [NB, Hkv, D, 16].

Sequence r's rows are its last cu[r + 1] - cu[r] positions; block tables map
positions to blocks.  Lengths come from the case (``lens``), so every seed of a
case does the same work.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False  # True: run() calls the framework's operators

BS = 16  # tokens per cache block
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
E_MIN, E_MAX = -100, 100
MIXED_CHUNK = 512  # tokens of a mixed launch's prefill chunks
VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]

# a drawn case costs no more than the largest listed ones
MOST_FLOPS, MOST_BYTES = 8e11, 4.5e8
# the plain attention's scores and gathered keys, as float32 values
MOST_SCORES, MOST_KEYS = 3.5e9, 1.2e9


def _attn(name, kind, seqs, prefix, ctx, q, heads=(32, 8, 128), prefixes=1, noalloc=False, lens=1):
    return {"name": name, "op": "attn", "cache": "kv4", "kind": kind, "hq": heads[0],
            "hkv": heads[1], "d": heads[2], "seqs": seqs, "prefix": prefix, "prefixes": prefixes,
            "ctx_lo": ctx[0], "ctx_hi": ctx[1], "q_lo": q[0], "q_hi": q[1], "noalloc": noalloc,
            "lens": lens}


def _rows(name, op, seqs, ctx, q, heads=(8, 128), dtype="bf16", lens=1):
    return {"name": name, "op": op, "cache": "kv4", "hkv": heads[0], "d": heads[1],
            "dtype": dtype, "seqs": seqs, "prefix": 0, "prefixes": 1, "ctx_lo": ctx[0],
            "ctx_hi": ctx[1], "q_lo": q[0], "q_hi": q[1], "lens": lens}


def _weights(name, seqs, ctx, q, cache="bf16", heads=(32, 8, 128), lens=1):
    return {"name": name, "op": "weights", "cache": cache, "hq": heads[0], "hkv": heads[1],
            "d": heads[2], "seqs": seqs, "prefix": 0, "prefixes": 1, "ctx_lo": ctx[0],
            "ctx_hi": ctx[1], "q_lo": q[0], "q_hi": q[1], "lens": lens}


def _evict(name, seqs, first, ctx, keep, window, cache="bf16", heads=(8, 128), lens=1):
    """``first`` tokens stay in front; of ``ctx`` behind them, the share ``keep`` in all."""
    return {"name": name, "op": "evict", "cache": cache, "hkv": heads[0], "d": heads[1],
            "seqs": seqs, "prefix": first, "prefixes": 1, "ctx_lo": ctx[0], "ctx_hi": ctx[1],
            "q_lo": 0, "q_hi": 0, "keep": keep, "window": window, "lens": lens}


def listed():
    return [
        # an interactive server: few requests in flight, latency of one layer, through
        # the entry point for callers that cannot allocate
        _attn("attn_decode_few", "decode", 4, 2048, (256, 1152), (1, 1), noalloc=True),
        # long private contexts that share nothing: all of the cache is read
        _attn("attn_decode_long", "decode", 24, 0, (8192, 20480), (1, 1), (64, 8, 128)),
        # new evidence of 32 requests against one cached prefix
        _attn("attn_prefill_batch", "prefill", 32, 2048, (0, 0), (256, 1024)),
        # chunked prefill and decode in one launch, a smaller model (head_dim 64)
        _attn("attn_mixed_d64", "mixed", 96, 1024, (256, 1152), (1, 1), (32, 8, 64), prefixes=2),
        # a decode step's new tokens, one for each request, most of them inside a block
        _rows("append_decode", "append", 256, (16, 1000), (1, 1)),
        # the prompts of a prefill step, on contexts that end anywhere in a block
        _rows("append_prefill", "append", 64, (0, 500), (256, 1024)),
        # one request's last few hundred tokens, in float32
        _rows("read_one", "read", 1, (100, 100), (389, 389), dtype="f32"),
        # whole contexts of 16 requests
        _rows("read_long", "read", 16, (0, 0), (4096, 12000)),
        # a decode step of 64 requests whose budget is counted at every token
        _weights("weights_decode", 64, (2048, 8192), (1, 1)),
        # the end of 16 long prompts judges what of them stays, over the 4-bit cache
        _weights("weights_window", 16, (4096, 12000), (64, 64), "kv4", (28, 4, 128)),
        # 64 requests of moderate length give half of their private context back
        _evict("evict_batch_kv4", 64, 512, (500, 1500), 0.5, 32, "kv4"),
        # 16 long contexts shrink to a quarter
        _evict("evict_long", 16, 64, (6000, 16000), 0.25, 256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["decode", "decode", "prefill", "verify", "mixed", "append", "append",
                       "read", "weights", "weights", "evict", "evict"])
    lens = rng.randrange(1 << 20)
    heads = rng.choice([(32, 8, 128), (28, 4, 128), (64, 8, 128), (32, 8, 64), (8, 2, 64)])
    prefix = rng.choice([0, _log(rng, 64, 4096), _log(rng, 512, 4096)])
    cache = rng.choice(["bf16", "kv4"])
    if what in ("append", "read"):
        hi, one = _log(rng, 1, 8192), rng.random() < 0.4
        lo = 1 if one else _log(rng, 1, 4096)
        c = _rows("", what, _log(rng, 1, 256), (rng.randint(0, hi), hi),
                  (lo, 1 if one else int(lo * rng.uniform(1, 4))), heads[1:],
                  rng.choice(["bf16", "bf16", "f32"]), lens=lens)
    elif what == "weights":
        lo, nq = _log(rng, 1, 8192), rng.choice([1, 1, _log(rng, 2, 64), _log(rng, 16, 1500)])
        c = _weights("", _log(rng, 1, 64), (lo, int(lo * rng.uniform(1, 3))),
                     (nq, int(nq * rng.uniform(1, 2))), cache, heads, lens=lens)
    elif what == "evict":
        lo = _log(rng, 32, 16384)
        c = _evict("", _log(rng, 1, 64), rng.choice([0, 4, _log(rng, 16, 2048)]),
                   (lo, int(lo * rng.uniform(1, 3))), rng.uniform(0.1, 0.9), _log(rng, 1, 256),
                   cache, heads[1:], lens=lens)
    elif what == "decode":
        lo = _log(rng, 1, 8192)
        c = _attn("", "decode", _log(rng, 1, 256), prefix, (lo, int(lo * rng.uniform(1, 3))),
                  (1, 1), heads, noalloc=rng.random() < 0.25, lens=lens)
    elif what == "prefill":
        lo = _log(rng, 1, 2048)
        c = _attn("", "prefill", _log(rng, 1, 32), prefix, (0, rng.choice([0, 512])),
                  (lo, int(lo * rng.uniform(1, 3))), heads, lens=lens)
    elif what == "verify":
        lo, nq = _log(rng, 16, 4096), rng.randint(2, 8)
        c = _attn("", "verify", _log(rng, 1, 32), prefix, (lo, int(lo * rng.uniform(1, 2))),
                  (nq, nq), heads, lens=lens)
    else:
        lo = _log(rng, 64, 512)
        c = _attn("", "mixed", _log(rng, 8, 96), _log(rng, 64, 1024), (lo, 4 * lo), (1, 1), heads,
                  prefixes=rng.randint(1, 3), lens=lens)
    del c["name"]
    while c["seqs"] > 1:
        w = work(c)
        fits = w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES
        sh = _shape(c)
        n, most = len(sh.q), max(sh.lens)
        if c["op"] in ("attn", "weights"):
            fits = (fits and n * max(sh.q) * c["hq"] * most <= MOST_SCORES
                    and n * most * c["hkv"] * c["d"] <= MOST_KEYS)
        if fits:
            break
        c["seqs"] = max(1, c["seqs"] * 3 // 4)
    return c


class _shape:
    """Lengths of a case's sequences: prefix of each, tokens cached behind it, new tokens."""

    def __init__(self, c):
        r = random.Random(c["lens"])
        self.plens = [c["prefix"] << p for p in range(c["prefixes"])]
        weights = [1.0 / (p + 1) ** 1.1 for p in range(c["prefixes"])]
        rows = []
        for i in range(c["seqs"]):
            p = r.choices(range(c["prefixes"]), weights)[0]
            if c.get("kind") == "mixed" and i % 8 == 0:
                rows.append((p, r.choice([0, MIXED_CHUNK]), MIXED_CHUNK))
            else:
                rows.append((p, r.randint(c["ctx_lo"], c["ctx_hi"]),
                             r.randint(c["q_lo"], c["q_hi"])))
        r.shuffle(rows)
        self.prefix = [p for p, _, _ in rows]
        self.ctx = [x for _, x, _ in rows]
        self.q = [q for _, _, q in rows]
        self.lens = [self.plens[p] + x + q for p, x, q in rows]
        self.total = sum(self.q)
        if c["op"] == "evict":
            first = c["prefix"]
            self.new = [first + max(1, int((L - first) * c["keep"])) for L in self.lens]


def _token_bytes(c):
    """Bytes of one token's key and value in the cache, all kv-heads."""
    if c["cache"] == "kv4":
        return c["hkv"] * (c["d"] + c["d"] // 32 + 1)
    return c["hkv"] * 4 * c["d"]


def work(c):
    sh = _shape(c)
    n, T, hkv, d, row = len(sh.q), sh.total, c["hkv"], c["d"], _token_bytes(c)
    meta = 4 * (sum(-(-x // BS) for x in sh.lens) + 2 * n)
    if c["op"] in ("append", "read"):
        # rows on one side, the cache's bytes on the other; an append's are read again,
        # as rows
        sides = 2 if c["op"] == "append" else 1
        return {"bytes": sides * T * (row + 2 * hkv * d * SIZE[c["dtype"]]) + 8 * n + 4 * T // BS,
                "flops": 2 * T * hkv * d}
    if c["op"] == "evict":
        kept, seen = sum(sh.new), sum(sh.lens)
        moved = sum(x - c["prefix"] // BS * BS for x in sh.new)
        # weights of all tokens, then the kept ones', their positions, keys and values
        return {"bytes": 4 * hkv * seen + 8 * hkv * kept + 2 * row * moved + meta,
                "flops": hkv * seen}
    cached = sum(sh.plens[p] // BS * BS for p in set(sh.prefix))
    cached += sum(L - sh.plens[p] // BS * BS for p, L in zip(sh.prefix, sh.lens))
    pairs = sum(q * (L - q) + q * (q + 1) // 2 for L, q in zip(sh.lens, sh.q))
    if c["op"] == "weights":
        keys = row * d // (2 * d) if c["cache"] == "bf16" else hkv * (d // 2 + d // 32)
        return {"bytes": cached * keys + T * c["hq"] * (2 * d + 4) + 4 * hkv * sum(sh.lens) + meta,
                "flops": 2 * d * c["hq"] * pairs}
    return {"bytes": cached * row + 4 * T * c["hq"] * d + 4 * T * c["hq"] + meta,
            "flops": 4 * d * c["hq"] * pairs}


# ---- the cache's numbers, in elementary operations -------------------------------------------

def _pow2(e):
    """2^e as float32, e of -126 .. 127 (integer tensor)."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _store4(x):
    """e2m1 codes and scale bytes of float32 x, the last dimension sharing a scale."""
    amax = x.abs().amax(-1)
    m, e = torch.frexp(amax)
    e = (e - 3 + (m > 0.875)).clamp(E_MIN, E_MAX)  # 7 = 0.875 2^3
    e = torch.where(amax > 0, e, E_MIN)
    y = (x * _pow2(-e)[..., None])
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5)
            + (a >= 3.5) + (a > 5))
    code |= y.view(torch.int32).lt(0).to(torch.uint8) << 3
    ok = torch.isfinite(amax)
    return torch.where(ok[..., None], code, 0), torch.where(ok, e + 127, 255).to(torch.uint8)


def _pack(code):
    """Pairs of neighbouring codes of the last dimension in bytes."""
    return code[..., 0::2] | code[..., 1::2] << 4


def _codes(x):
    """Codes of packed bytes, low halves first."""
    return torch.stack([x & 15, x >> 4], -1).flatten(-2)


def _numbers(x, scale):
    """float32 values of packed bytes; scale: its bytes, to broadcast."""
    table = torch.tensor(VALUES + [-v for v in VALUES], device=x.device)
    s = torch.where(scale == 255, math.nan, _pow2(scale.int().clamp(max=254) - 127))
    return table[_codes(x).int()] * s


def _value_rows(v):
    """[..., D / 32, 16, 16] bytes as [..., 16, D] codes."""
    code = _codes(v).unflatten(-1, (2, BS))     # [..., D / 32, 16 (i), 2 (a), 16 (o)]
    return code.movedim(-1, -4).transpose(-1, -2).flatten(-3)


def _value_blocks(code):
    """The inverse: codes [..., 16, D] as [..., D / 32, 16, 16] bytes."""
    x = code.unflatten(-1, (-1, 2, 16))         # [..., 16 (o), D / 32, 2, 16]
    return _pack(x.transpose(-1, -2).movedim(-4, -1).flatten(-2))


def _cached(st, block, offset=None):
    """float32 keys and values [..., D] of (block, offset), all kv-heads, or with no offset
    of whole blocks: [..., Hkv, 16, D]."""
    k, v = st["k_cache"], st["v_cache"]
    d = st["case"]["d"]
    if st["case"]["cache"] == "bf16":
        k, v = k[block], v[block]
        k = k.transpose(-3, -2).flatten(-2)[..., _key_slots(k.device), :]
        return k.float(), v.transpose(-1, -2).float()
    s = st["scales"]
    table = torch.tensor(VALUES + [-x for x in VALUES], device=v.device)
    if offset is None:
        s = s[block]
        k = _numbers(k[block].unflatten(-1, (d // 32, 16)),
                     s[..., :-1, :].transpose(-1, -2)[..., None])
        sv = _numbers(torch.full_like(s[..., -1, :], 2)[..., None], s[..., -1, :, None])[..., :1]
        return k.flatten(-2), table[_value_rows(v[block]).int()] * sv
    s = s[block, :, :, offset]                                    # [T, Hkv, D / 32 + 1]
    k = _numbers(k[block, :, offset].unflatten(-1, (d // 32, 16)), s[..., :-1, None]).flatten(-2)
    x = v.unflatten(-1, (2, 8))[block, :, :, :, :, offset // 2]   # [T, Hkv, D / 32, 16, 2]
    code = torch.where((offset % 2 == 1)[:, None, None, None, None], x >> 4, x & 15)
    sv = _numbers(torch.full_like(s[..., -1:], 2), s[..., -1:])[..., :1]
    return k, table[code.transpose(-1, -2).flatten(-3).int()] * sv


def _key_slots(device):
    """Slot of each offset in the bf16 cache's key blocks."""
    o = torch.arange(BS, device=device)
    return o & ~12 | (o & 4) << 1 | (o & 8) >> 1


# ---- inputs ----------------------------------------------------------------------------------

def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPE[c.get("dtype", "bf16")]

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, dtype=dtype, device="cuda", generator=gen)

    d, hkv, sh = c["d"], c["hkv"], _shape(c)
    n, T = len(sh.q), sh.total
    # block tables: a prefix's full blocks are shared, the rest is each sequence's own
    shared = [x // BS for x in sh.plens]
    private = [-(-L // BS) - shared[p] for p, L in zip(sh.prefix, sh.lens)]
    # blocks that an eviction's kept tokens go to
    fresh = [-(-x // BS) - shared[0] for x in sh.new] if c["op"] == "evict" else []
    nb = sum(shared) + sum(private) + sum(fresh) + 16
    ids = np.random.default_rng([seed, 1]).permutation(nb).astype(np.int32)
    start = np.concatenate([[0], np.cumsum(shared)])
    pblocks = [ids[start[p]:start[p + 1]] for p in range(len(shared))]

    def tables(counts, at):
        start = at + np.concatenate([[0], np.cumsum(counts)])
        table = np.full((n, max(shared[p] + x for p, x in zip(sh.prefix, counts))), -1, np.int32)
        for r, p in enumerate(sh.prefix):
            row = np.concatenate([pblocks[p], ids[start[r]:start[r + 1]]])
            table[r, :len(row)] = row
        return table

    table = tables(private, sum(shared))
    lens = np.array(sh.lens, np.int32)
    cu = np.concatenate([[0], np.cumsum(sh.q)]).astype(np.int32)
    st = {"case": c, "n": n, "total": T, "most_len": max(sh.lens), "most_q": max(sh.q),
          "block_table": torch.from_numpy(table).cuda(),
          "seq_lens": torch.from_numpy(lens).cuda(), "cu": torch.from_numpy(cu).cuda(),
          "scales": None}
    if c["cache"] == "bf16":
        st.update(k_cache=normal(nb, hkv, d // 32, BS, 32, dtype=torch.bfloat16),
                  v_cache=normal(nb, hkv, d, BS, dtype=torch.bfloat16))
    else:  # normal values whose spread differs from token to token, quantised in parts
        parts = [(_store4((normal(m, hkv, BS, d) * torch.exp(0.4 * normal(m, hkv, BS, 1)))
                          .unflatten(-1, (-1, 32))),
                  _store4(normal(m, hkv, BS, d) * torch.exp(0.4 * normal(m, hkv, BS, 1))))
                 for m in [4096] * (nb // 4096) + [nb % 4096] * (nb % 4096 > 0)]
        st.update(k_cache=torch.cat([_pack(k[0].flatten(-2)) for k, _ in parts]),
                  v_cache=torch.cat([_value_blocks(v[0]) for _, v in parts]),
                  scales=torch.cat([torch.cat([k[1].transpose(-1, -2), v[1][..., None, :]], -2)
                                    for k, v in parts]))
    if c["op"] in ("append", "read"):
        st.update(k_out=torch.empty((T, hkv, d), dtype=dt, device="cuda"),
                  v_out=torch.empty((T, hkv, d), dtype=dt, device="cuda"))
        if c["op"] == "append":  # some tokens are larger than others
            big = torch.exp(0.5 * normal(T, 1, 1))
            st.update(k_new=(normal(T, hkv, d) * big).to(dt),
                      v_new=(normal(T, hkv, d) * big).to(dt))
        return st
    if c["op"] == "evict":
        # a few tokens get most of the attention; small weights coincide now and then
        w = torch.exp(2 * normal(n, hkv, st["most_len"])) / 64
        st.update(weights=torch.round(w * 2 ** 20) / 2 ** 20, weights_out=torch.zeros_like(w),
                  kept=torch.full((n, hkv, max(sh.new)), -1, dtype=torch.int32, device="cuda"),
                  most_new=max(sh.new), new_table=torch.from_numpy(
                      tables(fresh, sum(shared) + sum(private))).cuda(),
                  new_lens=torch.tensor(sh.new, dtype=torch.int32).cuda(),
                  first=torch.full((n,), c["prefix"], dtype=torch.int32, device="cuda"))
        return st
    hq = c["hq"]
    st["q"] = normal(T, hq, d, dtype=torch.bfloat16)
    if c["op"] == "weights":
        # the attention call before has left the rows' log-sum-exp
        st["lse"] = torch.empty((T, hq), dtype=torch.float32, device="cuda")
        s, _ = _scores(st)
        top = s.amax(-1, keepdim=True)
        z = (top + s.sub_(top).exp_().sum(-1, keepdim=True).log()).squeeze(-1)
        z = z.permute(0, 2, 1, 3).reshape(n, st["most_q"], hq)
        st["lse"].copy_(z[_own_rows(st)])
        st["weights"] = torch.zeros((n, hkv, st["most_len"]), device="cuda")
        return st
    st.update(out=torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda"),
              lse=torch.empty((T, hq), dtype=torch.float32, device="cuda"))
    if own:  # the launch plan that a program builds once for all layers of a step
        from paper_2605_11232_amd import binding as B
        kind = {"decode": B.KIND_DECODE, "verify": B.KIND_VERIFY}.get(c["kind"], B.KIND_PREFILL)
        plan, info = B.plan(kind, sh.q[0] if c["kind"] == "verify" else 1, lens, cu, hq, hkv, d, BS,
                            B.PA_BF16_KV4, block_table=table)
        ws = torch.empty(int(info.workspace_bytes), dtype=torch.uint8, device="cuda")
        st.update(kind=kind, info=info, plan=torch.from_numpy(np.array(plan)).cuda(),
                  ws=ws if info.workspace_bytes else None)
    return st


# ---- one pass --------------------------------------------------------------------------------

def _positions(st):
    """Sequence and position of every row."""
    cu = st["cu"].long()
    seq = torch.repeat_interleave(torch.arange(st["n"], device="cuda"), cu[1:] - cu[:-1],
                                  output_size=st["total"])
    pos = torch.arange(st["total"], device="cuda") - cu[seq + 1] + st["seq_lens"][seq]
    return seq, pos


def _own_rows(st):
    """(sequence, row in it) of every row."""
    seq, pos = _positions(st)
    cu = st["cu"].long()
    return seq, pos - st["seq_lens"].long()[seq] + (cu[1:] - cu[:-1])[seq]


def _plain_append(st):
    c = st["case"]
    seq, pos = _positions(st)
    block, off = st["block_table"][seq, pos // BS].long(), pos % BS
    k, ks = _store4(st["k_new"].float().unflatten(-1, (-1, 32)))
    v, vs = _store4(st["v_new"].float())
    st["k_cache"][block, :, off] = _pack(k.flatten(-2))
    st["scales"][block, :, :, off] = torch.cat([ks, vs[..., None]], -1)
    # values: both halves of a byte may change, so first one, then the other
    cache = st["v_cache"].view(*st["v_cache"].shape[:4], 2, 8)
    v = v.unflatten(-1, (c["d"] // 32, 2, 16)).transpose(-1, -2)
    odd = (off % 2 == 1)[:, None, None, None, None]
    was = cache[block, :, :, :, :, off // 2]
    low = torch.where(odd, was, was & 0xF0 | v)
    even = torch.nonzero(off % 2 == 0).squeeze(1)
    cache[block[even], :, :, :, :, off[even] // 2] = low[even]
    was = cache[block, :, :, :, :, off // 2]
    high = was & 15 | v << 4
    o = torch.nonzero(off % 2 == 1).squeeze(1)
    cache[block[o], :, :, :, :, off[o] // 2] = high[o]
    _plain_read(st)


def _plain_read(st):
    seq, pos = _positions(st)
    k, v = _cached(st, st["block_table"][seq, pos // BS].long(), pos % BS)
    st["k_out"].copy_(k)
    st["v_out"].copy_(v)


def _scores(st):
    """Scaled scores [n, Hkv, most_q, G, keys], minus infinity where a row sees no key, and
    the values [n Hkv, keys, D]."""
    c = st["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    n, nq = st["n"], st["most_q"]
    L, cu = st["seq_lens"].long(), st["cu"].long()
    k, v = _cached(st, st["block_table"].long().clamp(min=0))          # [n, blocks, hkv, 16, D]
    k = k.permute(0, 2, 4, 1, 3).reshape(n * hkv, d, -1)              # [n hkv, D, keys]
    v = v.permute(0, 2, 1, 3, 4).reshape(n * hkv, -1, d)
    rows = (cu[:-1, None] + torch.arange(nq, device="cuda")).clamp(max=st["total"] - 1)
    q = st["q"][rows].float() * d ** -0.5                             # [n, nq, hq, D]
    q = q.view(n, nq, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(n * hkv, -1, d)
    s = torch.bmm(q, k).view(n, hkv, nq, hq // hkv, -1)
    last = (L - (cu[1:] - cu[:-1]))[:, None] + torch.arange(nq, device="cuda")
    last = torch.minimum(last, L[:, None] - 1)
    hidden = torch.arange(k.shape[2], device="cuda") > last[..., None]  # [n, nq, keys]
    s.masked_fill_(hidden[:, None, :, None], -math.inf)
    return s, v


def _plain_attention(st):
    c = st["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    n, nq = st["n"], st["most_q"]
    s, v = _scores(st)
    top = s.amax(-1, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(n * hkv, -1, p.shape[-1]), v).view(n, hkv, nq, hq // hkv, d)
    o = (o / total).permute(0, 2, 1, 3, 4).reshape(n, nq, hq, d)
    z = (top + total.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(n, nq, hq)
    at = _own_rows(st)
    st["out"].copy_(o[at].to(torch.bfloat16))
    st["lse"].copy_(z[at])


def _plain_weights(st):
    c = st["case"]
    hq, hkv, n, nq = c["hq"], c["hkv"], st["n"], st["most_q"]
    s, _ = _scores(st)
    cu = st["cu"].long()
    row = torch.arange(nq, device="cuda")
    z = st["lse"][(cu[:-1, None] + row).clamp(max=st["total"] - 1)]    # [n, nq, hq]
    z = torch.where((row < (cu[1:] - cu[:-1])[:, None])[..., None], z, math.inf)
    z = z.view(n, nq, hkv, hq // hkv).transpose(1, 2)
    w = s.sub_(z[..., None]).exp_().sum((2, 3))[..., :st["most_len"]]
    seen = torch.arange(st["most_len"], device="cuda") < st["seq_lens"][:, None, None]
    st["weights"].copy_(torch.where(seen, w, st["weights"]))


def _plain_evict(st):
    c = st["case"]
    w, L = st["weights"], st["seq_lens"].long()[:, None, None]
    new = torch.minimum(st["new_lens"].long()[:, None, None], L)
    first = torch.minimum(st["first"].long()[:, None, None], new)
    window = torch.clamp(new - first, max=c["window"])
    pos = torch.arange(w.shape[2], device="cuda")
    key = torch.where((pos < first) | (pos >= L - window), math.inf, w)
    key = torch.where(pos < L, key, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True)[1]
    stays = torch.zeros_like(key, dtype=torch.bool)
    stays.scatter_(2, order, (pos < new).expand_as(order))
    r, h, t = torch.nonzero(stays, as_tuple=True)
    to = (stays.cumsum(2) - 1)[r, h, t]
    st["kept"][r, h, to] = t.int()
    st["weights_out"][r, h, to] = w[r, h, t]
    # keys and values move to the new table's blocks
    a, x = st["block_table"][r, t // BS].long(), t % BS
    b, y = st["new_table"][r, to // BS].long(), to % BS
    k, v = st["k_cache"], st["v_cache"]
    if c["cache"] == "bf16":
        slot = _key_slots("cuda")
        k[b, h, :, slot[y]] = k[a, h, :, slot[x]]
        v[b, h, :, y] = v[a, h, :, x]
        return
    k[b, h, y] = k[a, h, x]
    st["scales"][b, h, :, y] = st["scales"][a, h, :, x]
    v = v.view(*v.shape[:4], 2, 8)
    code = v[a, h, :, :, :, x // 2] >> (4 * (x % 2)).to(torch.uint8)[:, None, None, None] & 15
    e = torch.nonzero(y % 2 == 0).squeeze(1)
    v[b[e], h[e], :, :, :, y[e] // 2] = v[b[e], h[e], :, :, :, y[e] // 2] & 0xF0 | code[e]
    o = torch.nonzero(y % 2 == 1).squeeze(1)
    v[b[o], h[o], :, :, :, y[o] // 2] = v[b[o], h[o], :, :, :, y[o] // 2] & 15 | code[o] << 4


def _own(st):
    from paper_2605_11232_amd import binding as B
    c = st["case"]
    op = c["op"]
    cache = st["k_cache"], st["v_cache"], st["scales"]
    where = st["block_table"], st["seq_lens"], st["cu"]
    if op == "append":
        B.kv4_append(st["k_new"], st["v_new"], *where, *cache)
    if op in ("append", "read"):
        B.kv4_read(st["k_out"], st["v_out"], *where, *cache)
    elif op == "weights":
        B.attention_weights(st["q"], st["lse"], st["k_cache"], *where, st["weights"],
                            scales=st["scales"])
    elif op == "evict":
        B.kv_evict(st["weights"], st["block_table"], st["seq_lens"], st["new_lens"],
                   st["k_cache"], st["v_cache"], st["kept"], scales=st["scales"],
                   new_table=st["new_table"], weights_out=st["weights_out"], first=st["first"],
                   window=c["window"])
    elif c["noalloc"] and st["info"].workspace_bytes <= B.NOALLOC_WORKSPACE_BYTES:
        B.kv4_attention_decode_noalloc(st["q"], *cache, *where, st["plan"], st["info"], st["out"],
                                       st["lse"])
    else:
        B.kv4_attention(st["kind"], st["q"], *cache, *where, st["plan"], st["info"], st["ws"],
                        st["out"], st["lse"])


def run(st):
    op = st["case"]["op"]
    if own:
        _own(st)
    else:
        {"append": _plain_append, "read": _plain_read, "attn": _plain_attention,
         "weights": _plain_weights, "evict": _plain_evict}[op](st)
    if op in ("append", "read"):
        return {"k": st["k_out"], "v": st["v_out"]}
    if op == "weights":
        return {"weights": st["weights"]}
    if op == "evict":  # what moved, as it lies in the caches
        out = {"kept": st["kept"], "weights": st["weights_out"], "k_cache": st["k_cache"],
               "v_cache": st["v_cache"]}
        if st["scales"] is not None:
            out["scales"] = st["scales"].view(torch.float8_e8m0fnu)
        return out
    return {"out": st["out"], "lse": st["lse"]}


# ---- 64 bits ---------------------------------------------------------------------------------

GRID = torch.tensor([-6, -4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6],
                    dtype=torch.float64)


def _nearest4(x):
    """Rows of x [..., dims that share a scale] as the cache holds them, in 64 bits: of two
    neighbours of the grid the nearer one; halfway the one whose place in it is even."""
    grid = GRID.to(x.device)
    s = torch.exp2(torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 7)).clamp(E_MIN, E_MAX))
    y = (x / s).clamp(-6, 6)
    hi = torch.searchsorted(grid, y.contiguous()).clamp(1, 14)
    lo = hi - 1
    below, above = y - grid[lo], grid[hi] - y
    # place 7 is zero: an odd distance from it is an odd code
    up = (above < below) | (above == below) & ((hi - 7) % 2 == 0)
    return torch.where(up, grid[hi], grid[lo]) * s


def _exact_codes(x):
    """e2m1 of codes, from the definition: 2^(exponent - 1) (1 + mantissa / 2)."""
    x = x.long()
    sign, e, m = 1 - 2 * (x >> 3).double(), x >> 1 & 3, (x & 1).double()
    return sign * torch.where(e == 0, m / 2, torch.exp2(e.double() - 1) * (1 + m / 2))


def _exact_cache(st, r, L):
    """Sequence r's keys and values in 64 bits, [Hkv, L, D]."""
    c = st["case"]
    hkv, d = c["hkv"], c["d"]
    b = st["block_table"][r, :-(-L // BS)].long()
    k, v = st["k_cache"][b], st["v_cache"][b]
    if c["cache"] == "bf16":
        k = torch.cat(k.double().unbind(2), -1)                  # [blocks, Hkv, slots, D]
        k = torch.cat([k[:, :, 0:4], k[:, :, 8:12], k[:, :, 4:8], k[:, :, 12:16]], 2)
        v = v.double().transpose(2, 3)
    else:
        s = torch.exp2(st["scales"][b].double() - 127)
        x = torch.empty((len(b), hkv, BS, d), dtype=torch.float64, device="cuda")
        x[..., 0::2], x[..., 1::2] = _exact_codes(k % 16), _exact_codes(k // 16)
        k = x * s[:, :, :-1].repeat_interleave(32, 2).transpose(2, 3)
        x = torch.empty_like(x)
        for i in range(d):  # dimension by dimension
            at = v[:, :, i // 32, i % 16, i // 16 % 2 * 8:i // 16 % 2 * 8 + 8]
            x[:, :, 0::2, i], x[:, :, 1::2, i] = _exact_codes(at % 16), _exact_codes(at // 16)
        v = x * s[:, :, -1, :, None]
    return (k.transpose(0, 1).reshape(hkv, -1, d)[:, :L],
            v.transpose(0, 1).reshape(hkv, -1, d)[:, :L])


def _exact_read(c, st):
    sh = _shape(c)
    if c["op"] == "append":
        k, v = st["k_new"].double(), st["v_new"].double()
        return {"k": torch.cat([_nearest4(x) for x in k.split(32, -1)], -1), "v": _nearest4(v)}
    rows = [[x[:, L - q:].transpose(0, 1) for x in _exact_cache(st, r, L)]
            for r, (L, q) in enumerate(zip(sh.lens, sh.q))]
    return {"k": torch.cat([k for k, _ in rows]), "v": torch.cat([v for _, v in rows])}


def _exact_attention(c, st):
    sh = _shape(c)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    out = torch.empty((sh.total, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((sh.total, hq), dtype=torch.float64, device="cuda")
    weights = torch.zeros((len(sh.q), hkv, max(sh.lens)), dtype=torch.float64, device="cuda")
    at = 0
    for r, (L, n) in enumerate(zip(sh.lens, sh.q)):
        k, v = _exact_cache(st, r, L)
        kt, v = k.transpose(1, 2).contiguous(), v.contiguous()
        many = max(1, (1 << 27) // (hq * L))  # queries at once: scores of at most 1 GiB
        for i in range(0, n, many):
            m = min(many, n - i)
            q = st["q"][at + i:at + i + m].double() / math.sqrt(d)
            q = q.view(m, hkv, hq // hkv, d).permute(1, 0, 2, 3).reshape(hkv, -1, d).contiguous()
            s = torch.bmm(q, kt).view(hkv, m, hq // hkv, L)
            last = torch.arange(L - n + i, L - n + i + m, device="cuda")
            s.masked_fill_((torch.arange(L, device="cuda") > last[:, None])[None, :, None],
                           -math.inf)
            if c["op"] == "weights":
                z = st["lse"][at + i:at + i + m].double().view(m, hkv, -1).transpose(0, 1)
                weights[r, :, :L] += torch.exp(s - z[..., None]).sum((1, 2))
                continue
            z = torch.logsumexp(s, 3)
            o = torch.bmm(s.sub_(z[..., None]).exp_().view(hkv, -1, L), v)
            out[at + i:at + i + m] = (o.view(hkv, m, hq // hkv, d).permute(1, 0, 2, 3)
                                      .reshape(m, hq, d))
            lse[at + i:at + i + m] = z.permute(1, 0, 2).reshape(m, hq)
        at += n
    return {"weights": weights} if c["op"] == "weights" else {"out": out, "lse": lse}


def _exact_evict(c, st):
    sh = _shape(c)
    w = st["weights"].double().cpu().numpy()
    out, kept = np.zeros(w.shape), st["kept"].cpu().numpy().astype(np.int64)
    for r, (L, B) in enumerate(zip(sh.lens, sh.new)):
        F = min(c["prefix"], B)
        W = min(c["window"], B - F)
        for h in range(c["hkv"]):
            x = w[r, h, F:L - W]
            heavy = np.lexsort((np.arange(len(x)), -x))[:B - F - W] + F
            at = np.concatenate([np.arange(F), np.sort(heavy), np.arange(L - W, L)])
            kept[r, h, :B], out[r, h, :B] = at, w[r, h, at]
    got = {"kept": torch.from_numpy(kept), "weights": torch.from_numpy(out), "k_cache": None,
           "v_cache": None}
    return got if c["cache"] == "bf16" else {**got, "scales": None}


def exact(c, seed):
    st = prepare(c, seed)
    return {"append": _exact_read, "read": _exact_read, "attn": _exact_attention,
            "weights": _exact_attention, "evict": _exact_evict}[c["op"]](c, st)
