"""Eviction from several contexts in one call where the pool has few free blocks, and from
contexts of which some are short enough to stay as they are."""
import numpy as np
import pytest
import torch

from paper_2605_11232_amd import binding as B
from tests.parity import say
from tests.test_gpu_evict import Session, cache_of, kept_of
from tests.test_gpu_kv8 import dev, tables

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


class TightSession(Session):
    """Contexts in a pool whose other blocks hold a finished request's prompt: they are cached
    and idle, all but `free` of them."""

    def __init__(self, cache, free, seed=0):
        super().__init__(cache, seed=seed)
        self.pool.set_eviction(True)
        other = (len(self.pool.free_list()) - free) * 16
        self.pool.add(99, [5000 + i for i in range(other)])
        self.pool.free(99)
        assert len(self.pool.free_list()) == free

    def shrink(self, new, first, window, in_place):
        m, _ = self.meta(self.ids, [0] * len(self.ids))
        old = m[0].copy()
        self.pool.compact_many(self.ids, new, [first] * len(new), in_place)
        after, _ = self.meta(self.ids, [0] * len(self.ids))
        keep = np.minimum(new, m[1])
        assert after[1].tolist() == keep.tolist()
        kept = torch.full((len(new), self.hkv, max(keep)), -1, dtype=torch.int32, device="cuda")
        B.kv_evict(self.weights, dev(old), dev(m[1]), dev(np.array(new, np.int32)), self.c.k, self.c.v,
                   kept, scales=self.c.scales, new_table=None if in_place else dev(after[0]),
                   first=dev(np.full(len(new), first, np.int32)), window=window)
        torch.cuda.synchronize()
        k = kept.cpu().numpy()
        for i, s in enumerate(self.ids):
            if new[i] >= m[1][i]:
                assert np.array_equal(after[0][i], old[i])
                assert np.array_equal(k[i, :, :keep[i]], np.tile(np.arange(keep[i]), (self.hkv, 1)))
            elif not in_place:
                assert not set(after[0][i, first // 16:]) - {-1} & set(old.reshape(-1))
            for store in (self.keys, self.values):
                store[s] = [store[s][h][k[i, h, :keep[i]]] for h in range(self.hkv)]


@pytest.mark.parametrize("free", [3, 14])
@pytest.mark.parametrize("cache", ["bf16", "kv4"])
def test_batch_where_free_blocks_are_few(cache, free):
    """Two of three contexts are shortened, together, to blocks that idle prompts give up; the
    third, with the shared prefix, stays.  The steps after it read what the call left."""
    say("[evict] few free blocks", cache, free)
    s = TightSession(cache, free)
    for _ in range(2):
        s.decode()
    s.shrink([200, 190, 200], 20, 8, False)
    assert s.pool.stats()["evictions"] > 0
    for _ in range(2):
        s.decode()
    s.shrink([90, 191, 100], 0, 5, False)
    s.decode()


@pytest.mark.parametrize("cache", ["bf16", "kv4"])
def test_no_blocks_for_a_batch_then_in_place(cache):
    """A refused batch leaves tables and contexts as they were, for an eviction in place."""
    say("[evict] no blocks for a batch", cache)
    s = TightSession(cache, 4)
    s.decode()
    s.pool.set_eviction(False)
    before = [s.pool.blocks_of(i) for i in s.ids], s.pool.free_list()
    with pytest.raises(B.PaError) as e:
        s.pool.compact_many(s.ids, [200, 200, 120], [96] * 3)
    assert e.value.code == "no_blocks"
    assert before == ([s.pool.blocks_of(i) for i in s.ids], s.pool.free_list())
    s.decode()
    s.shrink([200, 200, 200], 96, 8, True)
    s.decode()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("cache, d", [("bf16", 64), ("f32", 128), ("kv4", 128)])
def test_sequences_that_stay_share_their_blocks(cache, d, in_place):
    """Sequences of which all tokens stay have the same blocks in both tables, full ones of
    them shared with each other and, before what moves, with one that is shortened: no byte of
    them changes, positions and weights are written."""
    hkv, lens, new, first, window = 2, [100, 150, 64, 33, 300], [100, 999, 64, 40, 120], 64, 7
    say("[evict] sequences that stay", cache, d, in_place)
    r = np.random.default_rng(5)
    table, nb0 = tables(lens, 31)
    for i in range(1, 5):
        n = min(4, lens[i] // 16)
        table[i, :n] = table[0, :n]
    fresh, more = tables(lens, 32)
    to = table.copy()
    to[4, 4:] = np.where(fresh[4, 4:] >= 0, fresh[4, 4:] + nb0, -1)
    if in_place:
        to = table
    c = cache_of(cache, nb0 + more, hkv, d, 3)
    w = r.random((5, hkv, 300)).astype(np.float32)
    out = torch.full((5, hkv, 300), 7.0, device="cuda")
    kept = torch.full((5, hkv, 150), -5, dtype=torch.int32, device="cuda")
    before = [x.copy() for x in c.raw()]
    B.kv_evict(dev(w), dev(table), dev(np.array(lens, np.int32)), dev(np.array(new, np.int32)), c.k, c.v,
               kept, scales=c.scales, new_table=None if in_place else dev(to), weights_out=out,
               first=dev(np.full(5, first, np.int32)), window=window)
    torch.cuda.synchronize()
    want = [x.copy() for x in before]
    for i, L in enumerate(lens):
        b = min(new[i], L)
        for h in range(hkv):
            at = kept_of(w[i, h, :L].astype(np.float64), L, b, first, window)
            assert np.array_equal(kept[i, h].cpu().numpy(), np.concatenate([at, np.full(150 - b, -5)]))
            assert np.array_equal(out[i, h].cpu().numpy(),
                                  np.concatenate([w[i, h, at], np.full(300 - b, 7, np.float32)]))
            if i == 4:
                dst = np.arange(first, b)
                src = at[first:]
                for x, y in zip(want, before):
                    x[to[i, dst // 16], h, dst % 16] = y[table[i, src // 16], h, src % 16]
    for x, y in zip(c.raw(), want):
        assert np.array_equal(x, y)
