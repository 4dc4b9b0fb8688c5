"""Performance cases of the operators around the 8-bit KV cache.

Four operators, as one layer of a serving step calls them:

* ``rope``: queries and keys of the step's tokens, cut out of the projection's
  output, normalised for each head (root mean square, a weight per dimension)
  and rotated by their position.
* ``append``: the step's new keys and values quantised into the paged 8-bit
  cache.
* ``read``: tokens of the cache read back as rows, for a program that moves a
  context elsewhere or checks it.
* ``attn``: attention over the cache: prefill, decode, verification and the
  mixed launch.

The 8-bit cache holds e4m3 values and, for each (block, kv-head), a scale of
keys and one of values: powers of two 2^e, stored as the byte e + 127 (scales
[NB, Hkv, 2]).  Keys are [NB, Hkv, D / 64, 16, 64], values [NB, Hkv, D, 16].
A block's exponent is the smallest e of -100 .. 120 with amax <= 448 2^e over
its tokens' finite values.  An append to a block that holds earlier tokens
takes the larger of the block's exponent and the new tokens' one and rounds the
earlier tokens' values again where it grew.  Values that are not finite are
stored as NaN.  Rounding is to nearest even.

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
E_MIN, E_MAX = -100, 120
MIXED_CHUNK = 512  # tokens of a mixed launch's prefill chunks
N_POS = 32768      # positions of the rotation's table

# a drawn case costs no more than the largest listed ones
MOST_FLOPS, MOST_BYTES = 8e11, 7e8
# the plain attention's scores and gathered keys, as float32 values
MOST_SCORES, MOST_KEYS = 3.5e9, 1.2e9


def _attn(name, kind, seqs, prefix, ctx, q, heads=(32, 8, 128), prefixes=1, noalloc=False, lens=1):
    return {"name": name, "op": "attn", "kind": kind, "hq": heads[0], "hkv": heads[1],
            "d": heads[2], "seqs": seqs, "prefix": prefix, "prefixes": prefixes,
            "ctx_lo": ctx[0], "ctx_hi": ctx[1], "q_lo": q[0], "q_hi": q[1], "noalloc": noalloc,
            "lens": lens}


def _cache(name, op, seqs, ctx, q, heads=(8, 128), dtype="bf16", lens=1):
    return {"name": name, "op": op, "hkv": heads[0], "d": heads[1], "dtype": dtype, "seqs": seqs,
            "prefix": 0, "prefixes": 1, "ctx_lo": ctx[0], "ctx_hi": ctx[1], "q_lo": q[0],
            "q_hi": q[1], "lens": lens}


def _rope(name, tokens, heads=(32, 8, 128), rot=128, interleaved=False, norm=True, dtype="bf16"):
    return {"name": name, "op": "rope", "tokens": tokens, "hq": heads[0], "hkv": heads[1],
            "d": heads[2], "rot": rot, "interleaved": interleaved, "norm": norm, "dtype": dtype}


def listed():
    return [
        # an interactive server: few requests in flight, latency of one layer, through
        # the entry point for callers that cannot allocate
        _attn("attn_decode_few", "decode", 4, 2048, (256, 1152), (1, 1), noalloc=True),
        # the batch decode of the benchmark: 256 requests on one policy prefix
        _attn("attn_decode_batch", "decode", 256, 2048, (256, 1152), (1, 1)),
        # long private contexts that share nothing: all of the cache is read
        _attn("attn_decode_long", "decode", 24, 0, (8192, 20480), (1, 1), (64, 8, 128)),
        # new evidence of 32 requests against one cached prefix
        _attn("attn_prefill_batch", "prefill", 32, 2048, (0, 0), (256, 1024)),
        # chunked prefill and decode in one launch, a smaller model (head_dim 64)
        _attn("attn_mixed_d64", "mixed", 96, 1024, (256, 1152), (1, 1), (32, 8, 64), prefixes=2),
        # speculative verification on long contexts
        _attn("attn_verify", "verify", 24, 4096, (1024, 4096), (5, 5), (64, 8, 128)),
        # a decode step's new tokens, one for each request, most of them inside a block
        _cache("append_decode", "append", 256, (16, 1000), (1, 1)),
        # the prompts of a prefill step, on contexts that end anywhere in a block
        _cache("append_prefill", "append", 64, (0, 500), (256, 1024)),
        # one request's last few hundred tokens, in float32
        _cache("read_one", "read", 1, (100, 100), (389, 389), dtype="f32"),
        # whole contexts of 16 requests
        _cache("read_long", "read", 16, (0, 0), (4096, 12000)),
        # a decode step of 64 requests
        _rope("rope_decode", 64),
        # a prefill step; half of each head is rotated, in neighbouring pairs
        _rope("rope_prefill", 16384, rot=64, interleaved=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["decode", "decode", "prefill", "verify", "mixed", "append", "append",
                       "read", "rope", "rope"])
    lens = rng.randrange(1 << 20)
    heads = rng.choice([(32, 8, 128), (28, 4, 128), (64, 8, 128), (32, 8, 64), (8, 2, 64)])
    prefix = rng.choice([0, _log(rng, 64, 4096), _log(rng, 512, 4096)])
    if what == "rope":
        c = _rope("", _log(rng, 1, 20000), heads, rng.choice([heads[2], heads[2] // 2, 32, 6]),
                  rng.random() < 0.5, rng.random() < 0.8, rng.choice(["bf16", "bf16", "f32"]))
    elif what in ("append", "read"):
        hi, one = _log(rng, 1, 8192), rng.random() < 0.4
        lo = 1 if one else _log(rng, 1, 4096)
        c = _cache("", what, _log(rng, 1, 256), (rng.randint(0, hi), hi),
                   (lo, 1 if one else int(lo * rng.uniform(1, 4))), heads[1:],
                   rng.choice(["bf16", "bf16", "f32"]), lens=lens)
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
    while c.get("seqs", 1) > 1:
        w = work(c)
        fits = w["flops"] <= MOST_FLOPS and w["bytes"] <= MOST_BYTES
        if c["op"] == "attn":
            shape = _shape(c)
            n, most = len(shape.q), max(shape.lens)
            fits = (fits and n * max(shape.q) * c["hq"] * most <= MOST_SCORES
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


def work(c):
    if c["op"] == "rope":
        T, s = c["tokens"], SIZE[c["dtype"]]
        rows = T * (c["hq"] + c["hkv"]) * c["d"]
        table = min(T, N_POS) * c["rot"] * 4
        return {"bytes": 2 * rows * s + table + 4 * T + 2 * c["d"] * s,
                "flops": rows * (4 * c["norm"] + 3 * c["rot"] / c["d"])}
    sh = _shape(c)
    T, hkv, d = sh.total, c["hkv"], c["d"]
    row = 2 * hkv * d  # one token's keys and values in the cache
    meta = 4 * (sum(-(-x // BS) for x in sh.lens) + 2 * len(sh.q))
    if c["op"] != "attn":
        # rows on one side, the cache's bytes on the other, a scale pair per block and head
        blocks = sum((L - 1) // BS - (L - q) // BS + 1 for L, q in zip(sh.lens, sh.q))
        return {"bytes": T * row * (1 + SIZE[c["dtype"]]) + 2 * hkv * blocks + 8 * len(sh.q)
                + 4 * blocks, "flops": 2 * T * row}
    cached = sum(sh.plens[p] // BS * BS for p in set(sh.prefix))
    cached += sum(L - sh.plens[p] // BS * BS for p, L in zip(sh.prefix, sh.lens))
    flops = sum(4 * d * c["hq"] * (q * (L - q) + q * (q + 1) // 2) for L, q in zip(sh.lens, sh.q))
    return {"bytes": cached * (row + 2 * hkv / BS) + 4 * T * c["hq"] * d + 4 * T * c["hq"] + meta,
            "flops": flops}


# ---- the cache's numbers, in elementary operations -------------------------------------------

def _pow2(e):
    """2^e as float32, e of -126 .. 127 (integer tensor)."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _exponent(amax):
    """Smallest e of E_MIN .. E_MAX with amax <= 448 2^e (448 = 0.875 2^9)."""
    m, x = torch.frexp(amax)
    return (x - 9 + (m > 0.875)).clamp(E_MIN, E_MAX)


def _amax(x, dims):
    """Largest finite magnitude."""
    return torch.where(torch.isfinite(x), x.abs(), 0.0).amax(dims)


def _round8(x, e):
    """x / 2^e as e4m3; what is not finite as NaN."""
    return torch.where(torch.isfinite(x), x * _pow2(-e), math.nan).to(torch.float8_e4m3fn)


def _values(codes, scale):
    """Values a part of the cache stands for; scale: its bytes, to broadcast."""
    return codes.float() * _pow2(scale.int() - 127)


def _key_rows(k):
    """[..., D / 64, 16, 64] as [..., 16, D]."""
    return k.transpose(-3, -2).flatten(-2)


# ---- inputs ----------------------------------------------------------------------------------

def prepare(c, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPE[c.get("dtype", "bf16")]

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, dtype=dtype, device="cuda", generator=gen)

    d, hkv = c["d"], c["hkv"]
    if c["op"] == "rope":
        T, hq = c["tokens"], c["hq"]
        # the projection's output: queries, keys and values of a token side by side
        qkv = normal(T, hq + 2 * hkv, d).to(dt)
        freq = 10000.0 ** (-torch.arange(0, c["rot"], 2, dtype=torch.float64) / c["rot"])
        angle = torch.arange(N_POS, dtype=torch.float64)[:, None] * freq
        table = torch.cat([angle.cos(), angle.sin()], 1).float().cuda()
        pos = torch.randint(0, N_POS, (T,), device="cuda", generator=gen, dtype=torch.int32)
        st = {"case": c, "q": qkv[:, :hq], "k": qkv[:, hq:hq + hkv], "positions": pos,
              "table": table, "q_out": torch.empty((T, hq, d), dtype=dt, device="cuda"),
              "k_out": torch.empty((T, hkv, d), dtype=dt, device="cuda"),
              "q_weight": None, "k_weight": None}
        if c["norm"]:
            st["q_weight"] = (1 + 0.1 * normal(d)).to(dt)
            st["k_weight"] = (1 + 0.1 * normal(d)).to(dt)
        return st

    sh = _shape(c)
    n, T = len(sh.q), sh.total
    # block tables: a prefix's full blocks are shared, the rest is each sequence's own
    shared = [x // BS for x in sh.plens]
    private = [-(-L // BS) - shared[p] for p, L in zip(sh.prefix, sh.lens)]
    nb = sum(shared) + sum(private) + 16
    ids = np.random.default_rng([seed, 1]).permutation(nb).astype(np.int32)
    start = np.concatenate([[0], np.cumsum(shared)])
    pblocks = [ids[start[p]:start[p + 1]] for p in range(len(shared))]
    start = start[-1] + np.concatenate([[0], np.cumsum(private)])
    table = np.full((n, max(-(-L // BS) for L in sh.lens)), -1, np.int32)
    for r, p in enumerate(sh.prefix):
        row = np.concatenate([pblocks[p], ids[start[r]:start[r + 1]]])
        table[r, :len(row)] = row
    lens = np.array(sh.lens, np.int32)
    cu = np.concatenate([[0], np.cumsum(sh.q)]).astype(np.int32)

    # the cache: normal values whose spread differs from block to block, quantised
    def blocks(*shape):
        x = normal(nb, hkv, *shape)
        x *= torch.exp(0.4 * normal(nb, hkv, 1, 1))
        e = _exponent(_amax(x, (2, 3)))
        return _round8(x, e[:, :, None, None]), e

    k, ke = blocks(BS, d)
    v, ve = blocks(d, BS)
    k = k.view(torch.uint8).view(nb, hkv, BS, d // 64, 64).transpose(2, 3).contiguous()
    st = {"case": c, "n": n, "total": T, "most_len": max(sh.lens), "most_q": max(sh.q),
          "most_blocks": max((L - 1) // BS - (L - q) // BS + 1 for L, q in zip(sh.lens, sh.q)),
          "k_cache": k.view(torch.float8_e4m3fn), "v_cache": v,
          "scales": torch.stack([ke + 127, ve + 127], 2).to(torch.uint8),
          "block_table": torch.from_numpy(table).cuda(),
          "seq_lens": torch.from_numpy(lens).cuda(), "cu": torch.from_numpy(cu).cuda()}
    if c["op"] == "append":
        # some tokens are larger than all before them: their blocks' scales grow
        big = torch.exp(0.5 * normal(T, 1, 1))
        st.update(k_new=(normal(T, hkv, d) * big).to(dt), v_new=(normal(T, hkv, d) * big).to(dt))
    elif c["op"] == "read":
        st.update(k_out=torch.empty((T, hkv, d), dtype=dt, device="cuda"),
                  v_out=torch.empty((T, hkv, d), dtype=dt, device="cuda"))
    else:
        hq = c["hq"]
        st.update(q=normal(T, hq, d, dtype=torch.bfloat16),
                  out=torch.empty((T, hq, d), dtype=torch.bfloat16, device="cuda"),
                  lse=torch.empty((T, hq), dtype=torch.float32, device="cuda"))
        if own:  # the launch plan that a program builds once for all layers of a step
            from paper_2605_11232_amd import binding as B
            kind = {"decode": B.KIND_DECODE, "verify": B.KIND_VERIFY}.get(c["kind"],
                                                                         B.KIND_PREFILL)
            plan, info = B.plan(kind, sh.q[0] if c["kind"] == "verify" else 1, lens, cu, hq, hkv,
                                d, BS, B.PA_BF16_KV8, block_table=table)
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


def _plain_rope(st):
    c, table = st["case"], st["table"]
    ok = (st["positions"] >= 0) & (st["positions"] < len(table))
    cs = table[torch.where(ok, st["positions"], 0).long()][:, None]
    half = c["rot"] // 2
    cos, sin = cs[..., :half], cs[..., half:]

    def turn(x, w, out):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
        r, rest = x[..., :c["rot"]], x[..., c["rot"]:]
        if c["interleaved"]:
            a, b = r[..., 0::2], r[..., 1::2]
            r = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = r[..., :half], r[..., half:]
            r = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        y = torch.cat([r, rest], -1).to(out.dtype)
        out.copy_(torch.where(ok[:, None, None], y, out))

    turn(st["q"], st["q_weight"], st["q_out"])
    turn(st["k"], st["k_weight"], st["k_out"])


def _plain_append(st):
    L, cu = st["seq_lens"].long(), st["cu"].long()
    first = L - (cu[1:] - cu[:-1])  # first new position
    j = (first // BS)[:, None] + torch.arange(st["most_blocks"], device="cuda")
    seq, i = torch.nonzero((j * BS < L[:, None]) & (first < L)[:, None], as_tuple=True)
    j = j[seq, i]  # every (sequence, block) that gets new tokens
    block = st["block_table"][seq, j].long()
    pos = j[:, None] * BS + torch.arange(BS, device="cuda")
    old = pos < first[seq][:, None]
    new = ~old & (pos < L[seq][:, None])
    token = torch.where(new, cu[seq][:, None] + pos - first[seq][:, None], 0)

    def store(cache, side, x, to_rows, from_rows):
        was = to_rows(cache[block])                                  # [P, hkv, 16, D]
        scale = st["scales"][block, :, side]
        x = torch.where(new[:, None, :, None], x[token].float().transpose(1, 2), 0.0)
        e = _exponent(_amax(x, (2, 3)))
        e_old = scale.int() - 127
        e = torch.where(old.any(1)[:, None], torch.maximum(e, e_old), e)
        again = was.float() * _pow2((e_old - e).clamp(-126, 0))[..., None, None]
        code = torch.where(old[:, None, :, None], again.to(torch.float8_e4m3fn).view(torch.uint8),
                           was.view(torch.uint8))
        fresh = _round8(x, e[..., None, None]).view(torch.uint8)
        code = torch.where(new[:, None, :, None], fresh, code)
        cache.view(torch.uint8)[block] = from_rows(code)
        st["scales"][block, :, side] = (e + 127).to(torch.uint8)

    k, v = st["k_cache"], st["v_cache"]
    hkv, d = v.shape[1:3]
    store(k, 0, st["k_new"], _key_rows,
          lambda x: x.view(-1, hkv, BS, d // 64, 64).transpose(2, 3))
    store(v, 1, st["v_new"], lambda x: x.transpose(2, 3), lambda x: x.transpose(2, 3))


def _plain_read(st):
    seq, pos = _positions(st)
    block, off = st["block_table"][seq, pos // BS].long(), pos % BS
    scale = st["scales"][block]
    k = st["k_cache"][block, :, :, off].flatten(2)
    st["k_out"].copy_(_values(k, scale[..., 0:1]).to(st["k_out"].dtype))
    st["v_out"].copy_(_values(st["v_cache"][block, :, :, off], scale[..., 1:2])
                      .to(st["v_out"].dtype))


def _plain_attention(st):
    c = st["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    n, nq = st["n"], st["most_q"]
    L, cu = st["seq_lens"].long(), st["cu"].long()
    block = st["block_table"].long().clamp(min=0)
    scale = st["scales"][block]                                       # [n, blocks, hkv, 2]
    k = _values(_key_rows(st["k_cache"][block]), scale[..., 0, None, None])
    k = k.permute(0, 2, 4, 1, 3).reshape(n * hkv, d, -1)              # [n hkv, D, keys]
    v = _values(st["v_cache"][block], scale[..., 1, None, None])
    v = v.permute(0, 2, 1, 4, 3).reshape(n * hkv, -1, d)
    rows = (cu[:-1, None] + torch.arange(nq, device="cuda")).clamp(max=st["total"] - 1)
    q = st["q"][rows].float() * d ** -0.5                             # [n, nq, hq, D]
    q = q.view(n, nq, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(n * hkv, -1, d)
    s = torch.bmm(q, k).view(n, hkv, nq, hq // hkv, -1)
    last = (L - (cu[1:] - cu[:-1]))[:, None] + torch.arange(nq, device="cuda")
    last = torch.minimum(last, L[:, None] - 1)
    hidden = torch.arange(k.shape[2], device="cuda") > last[..., None]  # [n, nq, keys]
    s.masked_fill_(hidden[:, None, :, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(n * hkv, -1, p.shape[-1]), v).view(n, hkv, nq, hq // hkv, d)
    o = (o / total).permute(0, 2, 1, 3, 4).reshape(n, nq, hq, d)
    z = (top + total.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(n, nq, hq)
    seq, pos = _positions(st)
    i = pos - L[seq] + (cu[1:] - cu[:-1])[seq]
    st["out"].copy_(o[seq, i].to(torch.bfloat16))
    st["lse"].copy_(z[seq, i])


def _own(st):
    from paper_2605_11232_amd import binding as B
    op = st["case"]["op"]
    if op == "rope":
        B.qk_norm_rope(st["q"], st["k"], st["positions"], st["table"], st["q_out"], st["k_out"],
                       q_weight=st["q_weight"], k_weight=st["k_weight"], eps=1e-6,
                       norm=st["case"]["norm"], interleaved=st["case"]["interleaved"])
        return
    cache = st["k_cache"], st["v_cache"], st["scales"]
    where = st["block_table"], st["seq_lens"], st["cu"]
    if op == "append":
        B.kv8_append(st["k_new"], st["v_new"], *where, *cache)
    elif op == "read":
        B.kv8_read(st["k_out"], st["v_out"], *where, *cache)
    elif st["case"]["noalloc"] and st["info"].workspace_bytes <= B.NOALLOC_WORKSPACE_BYTES:
        B.kv8_attention_decode_noalloc(st["q"], *cache, *where, st["plan"], st["info"], st["out"],
                                       st["lse"])
    else:
        B.kv8_attention(st["kind"], st["q"], *cache, *where, st["plan"], st["info"], st["ws"],
                        st["out"], st["lse"])


def run(st):
    op = st["case"]["op"]
    if own:
        _own(st)
    else:
        {"rope": _plain_rope, "append": _plain_append, "read": _plain_read,
         "attn": _plain_attention}[op](st)
    if op == "rope":
        return {"q": st["q_out"], "k": st["k_out"]}
    if op == "append":  # the codes' values, and the powers of two that they are in
        return {"k_cache": st["k_cache"], "v_cache": st["v_cache"],
                "scales": st["scales"].view(torch.float8_e8m0fnu)}
    if op == "read":
        return {"k": st["k_out"], "v": st["v_out"]}
    return {"out": st["out"], "lse": st["lse"]}


# ---- 64 bits ---------------------------------------------------------------------------------

def _nearest8(x):
    """e4m3 of values up to 448, in 64 bits: multiples of 2^(exponent - 3), 2^-9 at least."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    # log2 may round up to a whole number just below one: its step is then too coarse
    step = torch.where(x.abs().clamp(min=2.0 ** -6) < 8 * step, step / 2, step)
    return torch.round(x / step) * step


def _exact_rope(c, st):
    half = c["rot"] // 2
    angle = st["table"].double()[st["positions"].long()]
    turn = torch.complex(angle[:, :half], angle[:, half:])[:, None]

    def of(x, w):
        x = x.double()
        if w is not None:
            x = x / (x.square().sum(-1, keepdim=True) / c["d"] + 1e-6).sqrt() * w.double()
        y = x[..., :c["rot"]]
        if c["interleaved"]:
            z = torch.view_as_complex(y.reshape(*y.shape[:-1], half, 2).contiguous()) * turn
            y = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(y[..., :half].contiguous(), y[..., half:].contiguous()) * turn
            y = torch.cat([z.real, z.imag], -1)
        return torch.cat([y, x[..., c["rot"]:]], -1)

    return {"q": of(st["q"], st["q_weight"]), "k": of(st["k"], st["k_weight"])}


def _exact_append(c, st):
    sh = _shape(c)
    out = {}
    for name, side, x in (("k_cache", 0, st["k_new"]), ("v_cache", 1, st["v_new"])):
        cache = st[name].double()
        if side == 0:  # as [NB, Hkv, 16, D]
            cache = torch.cat(cache.unbind(2), -1)
        else:
            cache = cache.transpose(2, 3).contiguous()
        scale = torch.exp2(st["scales"][:, :, side].double() - 127)
        at = 0
        for r, (L, q) in enumerate(zip(sh.lens, sh.q)):
            rows = x[at:at + q].double().transpose(0, 1)  # [hkv, q, D]
            at += q
            blocks = st["block_table"][r].long()
            pos = L - q
            # a block that holds earlier tokens, then whole blocks, then what is left
            done = 0
            while done < q:
                whole = (q - done) // BS if (pos + done) % BS == 0 else 0
                off = (pos + done) % BS
                n = whole * BS if whole else min(BS - off, q - done)
                b = blocks[(pos + done) // BS:(pos + done) // BS + max(whole, 1)]
                piece = rows[:, done:done + n].reshape(c["hkv"], len(b), -1, c["d"])
                piece = piece.transpose(0, 1)  # [blocks, hkv, tokens, D]
                need = piece.abs().amax((2, 3)) / 448
                s = torch.exp2(torch.ceil(torch.log2(need)).clamp(E_MIN, E_MAX))
                if off:
                    s = torch.maximum(s, scale[b])
                    cache[b, :, :off] = _nearest8(cache[b, :, :off]
                                                  * (scale[b] / s)[..., None, None])
                cache[b, :, off:off + piece.shape[2]] = _nearest8(piece / s[..., None, None])
                scale[b] = s
                done += n
        if side == 0:
            cache = torch.stack(cache.split(64, -1), 2)
        else:
            cache = cache.transpose(2, 3)
        out[name] = cache
        out.setdefault("scales", []).append(scale)
    out["scales"] = torch.stack(out["scales"], 2)
    return out


def _exact_cache(c, st, r, L):
    """Sequence r's keys and values in 64 bits, [Hkv, L, D]."""
    b = st["block_table"][r, :-(-L // BS)].long()
    scale = torch.exp2(st["scales"][b].double() - 127)[..., None, None]
    k = torch.cat(st["k_cache"][b].double().unbind(2), -1) * scale[:, :, 0]
    v = st["v_cache"][b].double().transpose(2, 3) * scale[:, :, 1]
    return (k.transpose(0, 1).reshape(c["hkv"], -1, c["d"])[:, :L],
            v.transpose(0, 1).reshape(c["hkv"], -1, c["d"])[:, :L])


def _exact_read(c, st):
    sh = _shape(c)
    rows = [[x[:, L - q:].transpose(0, 1) for x in _exact_cache(c, st, r, L)]
            for r, (L, q) in enumerate(zip(sh.lens, sh.q))]
    return {"k": torch.cat([k for k, _ in rows]), "v": torch.cat([v for _, v in rows])}


def _exact_attention(c, st):
    sh = _shape(c)
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    out = torch.empty((sh.total, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((sh.total, hq), dtype=torch.float64, device="cuda")
    at = 0
    for r, (L, n) in enumerate(zip(sh.lens, sh.q)):
        k, v = _exact_cache(c, st, r, L)
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
            z = torch.logsumexp(s, 3)
            o = torch.bmm(s.sub_(z[..., None]).exp_().view(hkv, -1, L), v)
            out[at + i:at + i + m] = (o.view(hkv, m, hq // hkv, d).permute(1, 0, 2, 3)
                                      .reshape(m, hq, d))
            lse[at + i:at + i + m] = z.permute(1, 0, 2).reshape(m, hq)
        at += n
    return {"out": out, "lse": lse}


def exact(c, seed):
    st = prepare(c, seed)
    return {"rope": _exact_rope, "append": _exact_append, "read": _exact_read,
            "attn": _exact_attention}[c["op"]](c, st)
