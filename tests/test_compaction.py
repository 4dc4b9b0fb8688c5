"""Compaction of several sequences at once, the pool's side of an eviction (CPU)."""
import numpy as np
import pytest

from oracle import apc
from paper_2605_11232_amd import binding as B

CODES = {"arg": apc.ArgError, "no_blocks": apc.NoBlocksError, "unknown_seq": apc.UnknownSeqError}


def state(pool, ids):
    return (pool.free_list(), pool.stats(), [(pool.blocks_of(s), pool.seq_len(s)) for s in ids])


@pytest.mark.parametrize("first", [0, 20, 32])
@pytest.mark.parametrize("cached", [False, True])
@pytest.mark.parametrize("evict", [False, True])
@pytest.mark.parametrize("spare", [0, 1, 3, 6, 9, 12])
def test_new_tables_have_no_block_of_an_old_one(spare, evict, cached, first):
    """Three contexts of 96 tokens to 48 in pools with few blocks or none besides theirs: one
    eviction call reads all old tables while it writes the new ones, from entry first / 16
    on.  Where blocks are too few, nothing changes."""
    nb = 18 + spare
    pool = B.Pool(nb, 16, np.random.default_rng(nb).permutation(nb).astype(np.int32), evict=evict)
    ids = [1, 2, 3]
    for s in ids:
        toks = [1000 * s + i for i in range(96)]
        pool.add(s, toks if cached else toks[:1])
        pool.extend(s, [] if cached else toks[1:])
    old = [pool.blocks_of(s) for s in ids]
    before = state(pool, ids)
    need = 3 * (3 - first // 16)
    if need > spare:
        with pytest.raises(B.PaError) as e:
            pool.compact_many(ids, [48] * 3, [first] * 3)
        assert e.value.code == "no_blocks"
        assert state(pool, ids) == before
        return
    pool.compact_many(ids, [48] * 3, [first] * 3)
    new = [pool.blocks_of(s) for s in ids]
    stay = first // 16
    got = [b for x in new for b in x[stay:]]
    assert len(got) == len(set(got)) == need
    assert not set(got) & {b for x in old for b in x}
    assert [x[:stay] for x in new] == [x[:stay] for x in old]
    assert [pool.seq_len(s) for s in ids] == [48] * 3
    # what was given back is there for later requests
    given = {b for x in old for b in x[stay:]}
    st = pool.stats()
    assert st["free_blocks"] + st["idle_cached_blocks"] == spare - need + len(given)
    assert (given <= set(pool.free_list())) == (not cached)


def test_idle_blocks_are_evicted_before_old_ones_come_back():
    """Blocks that the batch itself makes idle are not what it takes: those idle before are."""
    pool = B.Pool(22, 16, np.arange(22, dtype=np.int32), evict=True)
    pool.add(9, list(range(9000, 9064)))
    idle = pool.blocks_of(9)
    pool.free(9)
    for s in (1, 2):
        pool.add(s, [1000 * s + i for i in range(144)])
    old = {b for s in (1, 2) for b in pool.blocks_of(s)}
    assert pool.free_list() == [] and pool.stats()["idle_cached_blocks"] == 4
    pool.compact_many([1, 2], [32, 32])
    assert {b for s in (1, 2) for b in pool.blocks_of(s)} == set(idle)
    assert pool.stats()["evictions"] == 4 and pool.stats()["idle_cached_blocks"] == len(old)
    # their prompts still are
    assert pool.add(3, [1000 + i for i in range(144)]) == 128


@pytest.mark.parametrize("in_place", [False, True])
def test_short_sequences_stay_as_they_are(in_place):
    pool = B.Pool(40, 16, np.arange(40, dtype=np.int32))
    toks = {1: list(range(100)), 2: list(range(100, 148)), 3: list(range(200, 230))}
    for s, t in toks.items():
        pool.add(s, t[:1])
        pool.extend(s, t[1:])
    old = {s: pool.blocks_of(s) for s in toks}
    pool.compact_many([1, 2, 3], [48] * 3, None, in_place)
    assert [pool.seq_len(s) for s in (1, 2, 3)] == [48, 48, 30]
    assert [pool.blocks_of(s) for s in (2, 3)] == [old[2], old[3]]
    assert (pool.blocks_of(1) == old[1][:3]) == in_place
    for s in toks:
        pool.free(s)
    # a sequence that stayed is cached when it is freed, one that was shortened is not
    assert [pool.add(10 + s, toks[s] + [5] * 20) for s in (1, 2, 3)] == [0, 48, 16]


@pytest.mark.parametrize("in_place", [False, True])
def test_refusals_change_nothing(in_place):
    pool = B.Pool(60, 16, np.arange(60, dtype=np.int32))
    ids = [1, 2, 3]
    for s in ids:
        pool.add(s, [1000 * s + i for i in range(64)])
        pool.extend(s, list(range(40)))
    before = state(pool, ids)
    first = [64, 64, 64]
    for code, args in (("unknown_seq", ([1, 2, 4], [80] * 3, first)),
                       ("arg", ([1, 2, 1], [80] * 3, first)),
                       ("arg", ([1, 2, 2], [104] * 3, first)),
                       ("arg", (ids, [80, 80, 0], [64, 64, 0])),
                       ("arg", (ids, [80, 80, -1], first)),
                       ("arg", (ids, [80, 80, 80], [64, 64, 81])),
                       ("arg", (ids, [80, 80, 80], [64, 64, -1])),
                       ("arg", (ids, [80, 80, 104], [64, 64, -1]))):
        with pytest.raises(B.PaError) as e:
            pool.compact_many(*args, in_place)
        assert e.value.code == code and "pa_seqs_compact" in str(e.value)
        assert state(pool, ids) == before
    if in_place:  # blocks of a cached prompt would change, in the last of the batch
        with pytest.raises(B.PaError) as e:
            pool.compact_many(ids, [80] * 3, [64, 64, 63], True)
        assert e.value.code == "arg" and state(pool, ids) == before
    for bad in (([1, 2], [80] * 3, None), (ids, [80] * 3, [0, 0]), (ids, [80] * 2, None)):
        with pytest.raises(ValueError):
            pool.compact_many(*bad, in_place)
    lib = B.lib()
    assert lib.pa_seqs_compact(None, 0, None, None, None, 0) == B.PA_ERR_ARG
    assert lib.pa_seqs_compact(pool._h, -1, None, None, None, 0) == B.PA_ERR_ARG
    assert lib.pa_seqs_compact(pool._h, 1, None, None, None, 0) == B.PA_ERR_ARG
    assert lib.pa_seqs_compact(pool._h, 0, None, None, None, 0) == B.PA_OK
    assert state(pool, ids) == before
    pool.compact_many(ids, [80] * 3, first, in_place)
    assert [pool.seq_len(s) for s in ids] == [80] * 3


@pytest.mark.parametrize("evict", [False, True])
@pytest.mark.parametrize("seed", range(6))
def test_against_the_oracle(seed, evict):
    """Random admissions, extensions, releases and compactions of several sequences: the same
    blocks, free lists, counters and refusals; new tables are apart from all old ones."""
    r = np.random.default_rng([seed, 11])
    order = r.permutation(70).astype(np.int32)
    pool, orc = B.Pool(70, 4, order, evict=evict), apc.PrefixCacheOracle(70, 4, order)
    orc.evict = evict
    prefixes = [list(r.integers(0, 9, 24)) for _ in range(3)]
    live, next_id, refused, done = [], 0, 0, 0
    for _ in range(300):
        op = r.choice(["add", "add", "extend", "compact_many", "compact_many", "free"])
        sid = int(r.choice(live)) if live else 0
        if op == "add":
            sid, next_id = next_id, next_id + 1
            args = [sid, prefixes[r.integers(3)][:r.integers(1, 25)] + list(r.integers(0, 9, r.integers(0, 12)))]
        elif op == "extend":
            args = [sid, list(r.integers(0, 9, r.integers(0, 10)))]
        elif op == "compact_many":
            ids = [int(x) for x in r.permutation(live)[:r.integers(0, 5)]]
            if r.random() < 0.05:
                ids.append(ids[0] if ids and r.random() < 0.5 else next_id)
            n = [int(x) for x in r.integers(0 if r.random() < 0.1 else 1, 40, len(ids))]
            args = [ids, n, [int(r.integers(0, x + 1)) for x in n], bool(r.integers(2))]
            old = {b for s in live for b in pool.blocks_of(s)}
            tables = {s: (pool.blocks_of(s), pool.seq_len(s)) for s in live}
        else:
            args = [sid]
        want = None
        try:
            getattr(orc, {"free": "free_seq"}.get(op, op))(*args)
        except apc.OracleError as e:
            want = type(e)
        try:
            getattr(pool, op)(*args)
            assert want is None, (op, args)
        except B.PaError as e:
            refused += 1
            assert want is CODES[e.code], (op, args, e)
        if want is None and op in ("add", "free"):
            live = live + [sid] if op == "add" else [x for x in live if x != sid]
        if want is None and op == "compact_many":
            done += len(args[0])
            for s, n, front in zip(*args[:3]):
                was, length = tables[s]
                if n >= length:
                    assert pool.blocks_of(s) == was
                elif args[3]:
                    assert pool.blocks_of(s) == was[:-(-n // 4)]
                else:
                    assert not set(pool.blocks_of(s)[front // 4:]) & old
        assert pool.free_list() == orc.free_list() and pool.stats() == orc.stats()
        for x in live:
            assert pool.blocks_of(x) == orc.blocks_of(x) and pool.seq_len(x) == orc.seq_len(x)
    assert refused > 5 and done > 20
    for x in live:
        pool.free(x), orc.free_seq(x)
    assert pool.free_list() == orc.free_list() and pool.stats() == orc.stats()


def test_eviction_refuses_tables_of_no_blocks():
    """An empty tensor has no address; an eviction to it is not one in place."""
    import torch
    k = torch.zeros((4, 2, 4, 16, 32), dtype=torch.bfloat16)
    v = torch.zeros((4, 2, 128, 16), dtype=torch.bfloat16)
    bt, sl, nl = (torch.zeros(s, dtype=torch.int32) for s in ((1, 2), 1, 1))
    w, kept = torch.zeros((1, 2, 20)), torch.zeros((1, 2, 9), dtype=torch.int32)
    for tables in ((bt, torch.zeros((1, 0), dtype=torch.int32)), (bt[:, :0].contiguous(), None)):
        with pytest.raises(B.PaError) as e:
            B.kv_evict(w, tables[0], sl, nl, k, v, kept, new_table=tables[1])
        assert e.value.code == "arg" and "tables" in str(e.value)


@pytest.mark.parametrize("n, kept, blocks, w_stride, in_place", [
    (4096, 1 << 15, 2048, 4096, False), (4096, 1 << 20, 2048, 4096, False), (4096, 1 << 15, 4096, 4096, False),
    (1 << 19, 40, 3, 5000, False), (1 << 19, 40, 3, 100, True), (2**31 - 1, 2**62, 2**31 - 1, 1, False)])
def test_evictions_of_too_many_work_items_launch_nothing(n, kept, blocks, w_stride, in_place):
    """2^32 work-items or more in either launch, 4096 sequences of 8 kv-heads whose move would
    take four for each of 32768 tokens: refused before the selection changes the weights."""
    fn, lib = B.lib().pa_kv_evict, B.lib()
    assert fn(1 << 40, 1 << 40, w_stride, 64, 1 << 20, None if in_place else 128, blocks, 64, 64, None, 2,
              n, 1024, 2048, None, 16, 8, 128, 16, B.PA_BF16, 64, kept, None) == B.PA_ERR_LAUNCH
    assert b"invalid argument" in lib.pa_last_error(), lib.pa_last_error()
