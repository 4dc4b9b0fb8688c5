"""ctypes binding of libpa (include/pa.h): argument marshalling only.

Every computation runs in the C++/HIP library; this module converts numpy
arrays and torch tensors to pointers and return codes to exceptions.  If the
library is missing it raises -- there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpa.so")

PA_OK, PA_ERR_ARG, PA_ERR_UNSUPPORTED, PA_ERR_NO_BLOCKS, PA_ERR_UNKNOWN_SEQ, PA_ERR_LAUNCH = (
    0, -1, -2, -3, -4, -5)
PA_F32, PA_BF16, PA_BF16_KV8, PA_BF16_KV4 = 0, 1, 2, 4
QK_NORM, ROPE_INTERLEAVED = 1, 2
OP_ADD, OP_EXTEND, OP_TRUNCATE, OP_FREE = 0, 1, 2, 3
KIND_PREFILL, KIND_DECODE, KIND_VERIFY = 0, 1, 2
_CODES = {PA_ERR_ARG: "arg", PA_ERR_UNSUPPORTED: "unsupported", PA_ERR_NO_BLOCKS: "no_blocks",
          PA_ERR_UNKNOWN_SEQ: "unknown_seq", PA_ERR_LAUNCH: "launch"}

# Every symbol include/pa.h declares.
EXPORTS = ["pa_last_error", "pa_abi_version", "pa_pool_create", "pa_pool_destroy", "pa_seq_add",
           "pa_seq_extend", "pa_seq_truncate", "pa_seq_free", "pa_seqs_add", "pa_seqs_extend",
           "pa_seqs_truncate", "pa_seqs_free", "pa_pool_apply", "pa_seq_len", "pa_seq_blocks",
           "pa_pool_free_list", "pa_build_metadata", "pa_attn_plan", "pa_kv_append",
           "pa_attn_prefill", "pa_attn_decode", "pa_attn_verify", "pa_pool_set_eviction",
           "pa_pool_get_stats", "pa_pool_kv_waste", "pa_form_batches", "pa_prepare_launch",
           "pa_stage_upload", "pa_attn_workspace_size", "pa_attn_decode_workspace_size",
           "pa_attn_decode_noalloc", "pa_kv8_append", "pa_kv8_read", "pa_kv8_attn_prefill",
           "pa_kv8_attn_decode", "pa_kv8_attn_verify", "pa_kv8_attn_decode_noalloc",
           "pa_kv4_append", "pa_kv4_read", "pa_kv4_attn_prefill", "pa_kv4_attn_decode",
           "pa_kv4_attn_verify", "pa_kv4_attn_decode_noalloc",
           "pa_seq_compact", "pa_seqs_compact", "pa_attn_weights", "pa_kv_evict", "pa_qk_norm_rope",
           "pa_set_launch_events"]


class PaError(RuntimeError):
    def __init__(self, rc: int, msg: str):
        super().__init__(f"[{_CODES.get(rc, rc)}] {msg}")
        self.rc = rc
        self.code = _CODES.get(rc, str(rc))


class PoolStats(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("num_blocks", "free_blocks", "cached_blocks",
                                         "idle_cached_blocks", "evictions", "live_seqs",
                                         "live_tokens", "logical_blocks", "physical_blocks")]


class KvWaste(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("paged_slots", C.c_int64), ("physical_slots", C.c_int64),
                ("contiguous_slots", C.c_int64), ("paged_waste", C.c_double),
                ("contiguous_waste", C.c_double), ("sharing_factor", C.c_double)]


class PlanInfo(C.Structure):
    _fields_ = [("kind", C.c_int32), ("n_q", C.c_int32), ("n_shared_items", C.c_int32),
                ("n_tile_items", C.c_int32), ("n_row_items", C.c_int32), ("n_groups", C.c_int32),
                ("n_merge_rows", C.c_int32), ("grid", C.c_int32), ("variant", C.c_int32),
                ("n_merge_items", C.c_int32), ("plan_words", C.c_int64), ("workspace_bytes", C.c_int64),
                ("n_seqs", C.c_int32), ("total_q", C.c_int32), ("num_q_heads", C.c_int32),
                ("num_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("partial_rows", C.c_int64)]


_lib = None
_torch = None  # the torch module, once a call needed it
_attn = {}     # attention entry point of each launch kind
_kv8_attn = {}  # and over the 8-bit cache
_kv4_attn = {}  # and over the 4-bit cache
_ROW_DTYPES = {}  # dtype codes of rows, once torch is there
_P = C.c_void_p
_I32P = C.POINTER(C.c_int32)
_I64P = C.POINTER(C.c_int64)


def lib():
    """Load libpa.so (built in-tree by ``paper_2605_11232_amd.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2605_11232_amd.build` (no fallback exists)")
    L = C.CDLL(LIB_PATH)
    i32, i64, f32 = C.c_int32, C.c_int64, C.c_float
    sig = {
        "pa_last_error": (C.c_char_p, []),
        "pa_abi_version": (i32, []),
        "pa_pool_create": (C.c_int, [i32, i32, _I32P, C.POINTER(_P)]),
        "pa_pool_destroy": (None, [_P]),
        "pa_seq_add": (C.c_int, [_P, i64, _I32P, i32, _I32P]),
        "pa_seq_extend": (C.c_int, [_P, i64, _I32P, i32]),
        "pa_seq_truncate": (C.c_int, [_P, i64, i32]),
        "pa_seq_free": (C.c_int, [_P, i64]),
        "pa_seqs_add": (C.c_int, [_P, i32, _I64P, _I32P, _I32P, _I32P, _I32P]),
        "pa_seqs_extend": (C.c_int, [_P, i32, _I64P, _I32P, _I32P, _I32P]),
        "pa_seqs_truncate": (C.c_int, [_P, i32, _I64P, _I32P, _I32P]),
        "pa_seqs_free": (C.c_int, [_P, i32, _I64P, _I32P]),
        "pa_seq_compact": (C.c_int, [_P, i64, i32, i32, i32]),
        "pa_seqs_compact": (C.c_int, [_P, i32, _I64P, _I32P, _I32P, i32]),
        "pa_pool_apply": (C.c_int, [_P, i32, _P, _P, _P, _P, _P, _P, _P]),
        "pa_seq_len": (C.c_int, [_P, i64, _I32P]),
        "pa_seq_blocks": (C.c_int, [_P, i64, _I32P, i32, _I32P]),
        "pa_pool_free_list": (C.c_int, [_P, _I32P, i32, _I32P]),
        "pa_build_metadata": (C.c_int, [_P, i32, _I64P, _I32P, i32, _I32P, _I32P, _I32P, _I32P, i64]),
        "pa_attn_plan": (C.c_int, [i32, i32, i32, _I32P, _I32P, _I32P, i32, i32, i32, i32, i32, i32,
                                   i32, _I32P, i64, C.POINTER(PlanInfo)]),
        "pa_kv_append": (C.c_int, [_P, _P, _P, i32, _P, _P, i32, i32, i32, i32, i32, _P]),
        "pa_stage_upload": (C.c_int, [_P, _P, i64, _P]),
        "pa_attn_workspace_size": (C.c_int, [i32, i32, i32, i32, C.POINTER(C.c_size_t)]),
        "pa_attn_decode_workspace_size": (C.c_int, [i32, i32, i32, i32, C.POINTER(C.c_size_t)]),
        "pa_pool_set_eviction": (C.c_int, [_P, i32]),
        "pa_pool_get_stats": (C.c_int, [_P, C.POINTER(PoolStats)]),
        "pa_pool_kv_waste": (C.c_int, [_P, i32, C.POINTER(KvWaste)]),
        "pa_form_batches": (C.c_int, [i32, _I32P, _I32P, i32, _I32P, _I32P, _I32P, _I32P, _I32P,
                                      _I32P, _I32P]),
        "pa_prepare_launch": (C.c_int, [_P, i32, _P, _P, _P, _P, _P, _P, i32, _P, _P, i32, _P, _P,
                                        _P, _P, i64, i32, i32, i32, i32, i32, i32, i32, i32, _P,
                                        i64, C.POINTER(PlanInfo)]),
    }
    attn = (C.c_int, [_P, _P, _P, i32, _P, i32, _P, _P, i32, i32, i32, i32, i32, i32, f32, i32, _P,
                      C.POINTER(PlanInfo), _P, C.c_size_t, _P, _P, _P])
    for name in ("pa_attn_prefill", "pa_attn_decode", "pa_attn_verify"):
        sig[name] = attn
    # decode without the workspace pair
    sig["pa_attn_decode_noalloc"] = (C.c_int, attn[1][:18] + attn[1][20:])
    rows = [_P, i64, _P, i64, _P, i32, _P, _P, i32, i32, _P, _P, _P, i32, i32, i32, i32, i32, _P]
    for name in ("pa_kv8_append", "pa_kv8_read", "pa_kv4_append", "pa_kv4_read"):
        sig[name] = (C.c_int, rows)
    # the scales behind the caches, and no dtype
    kv8 = attn[1][:3] + [_P] + attn[1][3:15] + attn[1][16:]
    for bits in ("8", "4"):
        for kind in ("prefill", "decode", "verify"):
            sig[f"pa_kv{bits}_attn_{kind}"] = (C.c_int, kv8)
        sig[f"pa_kv{bits}_attn_decode_noalloc"] = (C.c_int, kv8[:18] + kv8[20:])
    sig["pa_attn_weights"] = (C.c_int, [_P, _P, _P, _P, i32, _P, i32, _P, _P, i32, i32, i32, i32,
                                        i32, i32, f32, i32, _P, i64, i32, _P])
    sig["pa_kv_evict"] = (C.c_int, [_P, _P, i64, _P, i32, _P, i32, _P, _P, _P, i32, i32, _P, _P, _P,
                                    i32, i32, i32, i32, i32, _P, i64, _P])
    sig["pa_qk_norm_rope"] = (C.c_int, [_P, i64, _P, i64, _P, i32, _P, i32, i32, _P, _P, f32, i32,
                                        _P, _P, i32, i32, i32, i32, _P])
    sig["pa_set_launch_events"] = (C.c_int, [_P, _P])
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _attn.update({KIND_PREFILL: L.pa_attn_prefill, KIND_DECODE: L.pa_attn_decode,
                  KIND_VERIFY: L.pa_attn_verify})
    _kv8_attn.update({KIND_PREFILL: L.pa_kv8_attn_prefill, KIND_DECODE: L.pa_kv8_attn_decode,
                      KIND_VERIFY: L.pa_kv8_attn_verify})
    _kv4_attn.update({KIND_PREFILL: L.pa_kv4_attn_prefill, KIND_DECODE: L.pa_kv4_attn_decode,
                      KIND_VERIFY: L.pa_kv4_attn_verify})
    _lib = L
    return L


def _check(rc: int):
    if rc != PA_OK:
        raise PaError(rc, lib().pa_last_error().decode())


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.int32)


def _ptr(a: np.ndarray, ctype=C.c_int32):
    return a.ctypes.data_as(C.POINTER(ctype))


def _addr(a) -> int:
    """Address of a numpy array's data (0 for None or an empty array)."""
    return 0 if a is None or a.size == 0 else a.ctypes.data


class PackedOps:
    """A step's pool operations as pa_pool_apply takes them (ops, seq_ids,
    token_offsets, tokens, new_lens), plus the n_cached output array, with
    their addresses taken once so that repeated calls marshal nothing."""

    def __init__(self, ops, seq_ids, offsets, tokens, new_lens):
        self.ops = _i32(ops)
        self.seq_ids = np.ascontiguousarray(seq_ids, dtype=np.int64)
        self.offsets = _i32(offsets)
        self.tokens = _i32(tokens)
        self.new_lens = _i32(new_lens)
        self.n = int(self.ops.size)
        if not (self.seq_ids.size == self.n and self.offsets.size == self.n + 1
                and self.new_lens.size == self.n):
            raise ValueError("PackedOps: arrays of inconsistent length")
        self.n_cached = np.zeros(max(1, self.n), np.int32)
        self.addrs = (_addr(self.ops), _addr(self.seq_ids), _addr(self.offsets),
                      _addr(self.tokens), _addr(self.new_lens), _addr(self.n_cached))
        self.add_rows = np.flatnonzero(self.ops == OP_ADD)
        self.add_ids = self.seq_ids[self.add_rows].tolist()

    def admitted(self) -> dict:
        """{seq_id: reused tokens} of the admissions of the last application."""
        return dict(zip(self.add_ids, self.n_cached[self.add_rows].tolist())) if self.add_ids else {}


class LaunchInputs:
    """One launch's sequence ids (int64) and query lengths (int32), with
    their addresses taken once."""

    def __init__(self, seq_ids, q_lens):
        self.seq_ids = np.ascontiguousarray(seq_ids, dtype=np.int64)
        self.q_lens = _i32(q_lens)
        if self.seq_ids.size != self.q_lens.size:
            raise ValueError("LaunchInputs: seq_ids and q_lens differ in length")
        self.n = int(self.seq_ids.size)
        self.total_q = int(self.q_lens.sum()) if self.n else 0
        self.addrs = (_addr(self.seq_ids), _addr(self.q_lens))


class LaunchBuffers:
    """Caller-owned host int32 arrays that launch metadata and plan are
    written to (e.g. views of one pinned staging buffer): block_table
    [rows, max_blocks], seq_lens [rows], cu_seqlens_q [rows + 1],
    slot_mapping [tokens], plan [words]; addresses taken once."""

    def __init__(self, block_table, seq_lens, cu_seqlens_q, slot_mapping, plan):
        arrs = (block_table, seq_lens, cu_seqlens_q, slot_mapping, plan)
        for a in arrs:
            if a.dtype != np.int32 or not a.flags["C_CONTIGUOUS"]:
                raise ValueError("LaunchBuffers: arrays must be contiguous int32")
        if block_table.ndim != 2 or seq_lens.size != block_table.shape[0] or \
                cu_seqlens_q.size < seq_lens.size + 1:
            raise ValueError("LaunchBuffers: inconsistent shapes")
        self.block_table, self.seq_lens, self.cu_seqlens_q, self.slot_mapping, self.plan = arrs
        self.rows, self.max_blocks = (int(x) for x in block_table.shape)
        # slot_mapping may be empty; a non-null address is passed regardless
        self.addrs = tuple(a.ctypes.data for a in arrs)

    def meta(self, n: int, total_q: int) -> dict:
        """Views of the first launch's metadata (as Pool.metadata returns)."""
        return {"block_table": self.block_table[:n], "seq_lens": self.seq_lens[:n],
                "cu_seqlens_q": self.cu_seqlens_q[:n + 1],
                "slot_mapping": self.slot_mapping[:total_q]}


class Pool:
    """Host block manager (prefix-hit lookup, allocation, tables, slots)."""

    def __init__(self, num_blocks: int, block_size: int, free_order, evict: bool = False):
        self._lib = lib()
        fo = _i32(free_order)
        h = _P()
        _check(self._lib.pa_pool_create(int(num_blocks), int(block_size),
                                        _ptr(fo) if fo.size else None, C.byref(h)))
        self._h = h
        self.num_blocks, self.block_size = int(num_blocks), int(block_size)
        if evict:
            self.set_eviction(True)

    def set_eviction(self, enabled: bool):
        _check(self._lib.pa_pool_set_eviction(self._h, int(bool(enabled))))

    def stats(self) -> dict:
        st = PoolStats()
        _check(self._lib.pa_pool_get_stats(self._h, C.byref(st)))
        return {n: int(getattr(st, n)) for n, _ in PoolStats._fields_}

    def kv_waste(self, max_seq_len: int) -> dict:
        w = KvWaste()
        _check(self._lib.pa_pool_kv_waste(self._h, int(max_seq_len), C.byref(w)))
        return {n: (float if t is C.c_double else int)(getattr(w, n)) for n, t in KvWaste._fields_}

    def close(self):
        if getattr(self, "_h", None):
            self._lib.pa_pool_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def add(self, seq_id: int, tokens) -> int:
        t = _i32(tokens)
        n = C.c_int32(0)
        _check(self._lib.pa_seq_add(self._h, int(seq_id), _ptr(t) if t.size else None, t.size,
                                    C.byref(n)))
        return n.value

    def extend(self, seq_id: int, tokens):
        t = _i32(tokens)
        _check(self._lib.pa_seq_extend(self._h, int(seq_id), _ptr(t) if t.size else None, t.size))

    def truncate(self, seq_id: int, new_len: int):
        _check(self._lib.pa_seq_truncate(self._h, int(seq_id), int(new_len)))

    def compact(self, seq_id: int, new_len: int, first: int = 0, in_place: bool = False):
        """The pool's side of a kv_evict of this sequence alone: it holds new_len tokens, its
        first ``first`` ones unchanged, in new blocks or (``in_place``) in its own.  Calls
        that follow may hand out the blocks that it gives back: one kv_evict for several
        sequences needs compact_many."""
        _check(self._lib.pa_seq_compact(self._h, int(seq_id), int(new_len), int(first),
                                        int(bool(in_place))))

    def free(self, seq_id: int):
        _check(self._lib.pa_seq_free(self._h, int(seq_id)))

    # -- batched forms (one library call per serving step) --------------------
    def add_many(self, seq_ids, offsets, tokens):
        """Admit len(seq_ids) sequences; returns reused-token counts (int32)."""
        ids = np.ascontiguousarray(seq_ids, dtype=np.int64)
        off, tok = _i32(offsets), _i32(tokens)
        out = np.zeros(ids.size, np.int32)
        _check(self._lib.pa_seqs_add(self._h, ids.size, ids.ctypes.data_as(_I64P), _ptr(off),
                                     _ptr(tok) if tok.size else None, _ptr(out), None))
        return out

    def extend_many(self, seq_ids, offsets, tokens):
        ids = np.ascontiguousarray(seq_ids, dtype=np.int64)
        off, tok = _i32(offsets), _i32(tokens)
        _check(self._lib.pa_seqs_extend(self._h, ids.size, ids.ctypes.data_as(_I64P), _ptr(off),
                                        _ptr(tok) if tok.size else None, None))

    def truncate_many(self, seq_ids, new_lens):
        ids = np.ascontiguousarray(seq_ids, dtype=np.int64)
        nl = _i32(new_lens)
        _check(self._lib.pa_seqs_truncate(self._h, ids.size, ids.ctypes.data_as(_I64P), _ptr(nl),
                                          None))

    def compact_many(self, seq_ids, new_lens, first=None, in_place: bool = False):
        """The pool's side of one kv_evict for these sequences (first: an array, or None for
        none): all of them or, where it raises, none; those of new_lens tokens or fewer stay
        as they are."""
        ids = np.ascontiguousarray(seq_ids, dtype=np.int64)
        nl, fr = _i32(new_lens), None if first is None else _i32(first)
        if nl.shape != ids.shape or (fr is not None and fr.shape != ids.shape):
            raise ValueError("compact_many: arrays of inconsistent length")
        _check(self._lib.pa_seqs_compact(self._h, ids.size, ids.ctypes.data_as(_I64P), _ptr(nl),
                                         None if fr is None else _ptr(fr), int(bool(in_place))))

    def free_many(self, seq_ids):
        ids = np.ascontiguousarray(seq_ids, dtype=np.int64)
        _check(self._lib.pa_seqs_free(self._h, ids.size, ids.ctypes.data_as(_I64P), None))

    def apply(self, ops, seq_ids, offsets, tokens, new_lens):
        """Mixed pool operations in one call (arrays as pa_pool_apply takes
        them); returns reused-token counts (int32, 0 for non-admissions)."""
        p = PackedOps(ops, seq_ids, offsets, tokens, new_lens)
        return self.apply_packed(p).copy()

    def apply_packed(self, p: PackedOps):
        """pa_pool_apply on pre-packed operations; returns p's n_cached view."""
        if p.n:
            _check(self._lib.pa_pool_apply(self._h, p.n, *p.addrs, None))
        return p.n_cached[:p.n]

    def prepare_launch(self, ops, inp: LaunchInputs, buf: LaunchBuffers, kind: int, n_q: int,
                       num_q_heads: int, num_kv_heads: int, head_dim: int, dtype: int,
                       num_cus: int = 0, shared_prefix: bool = True, info=None):
        """pa_prepare_launch: ``ops`` (PackedOps or None) applied, then the
        metadata of ``inp`` and its plan written into ``buf``; returns the
        PlanInfo (``info`` is reused when given)."""
        if inp.n > buf.rows or inp.total_q > buf.slot_mapping.size:
            raise ValueError("prepare_launch: launch larger than its buffers")
        if info is None:
            info = PlanInfo()
        if ops is not None and ops.n:
            n_ops, oa = ops.n, ops.addrs
        else:
            n_ops, oa = 0, (0, 0, 0, 0, 0, 0)
        bt, sl, cu, sm, pl = buf.addrs
        _check(self._lib.pa_prepare_launch(
            self._h, n_ops, *oa, inp.n, *inp.addrs, buf.max_blocks, bt, sl, cu, sm,
            buf.slot_mapping.size, int(kind), int(n_q), int(num_q_heads), int(num_kv_heads),
            int(head_dim), int(dtype), int(num_cus), 1 if shared_prefix else 0, pl,
            buf.plan.size, C.byref(info)))
        return info

    def seq_len(self, seq_id: int) -> int:
        n = C.c_int32(0)
        _check(self._lib.pa_seq_len(self._h, int(seq_id), C.byref(n)))
        return n.value

    def blocks_of(self, seq_id: int):
        n = C.c_int32(0)
        rc = self._lib.pa_seq_blocks(self._h, int(seq_id), None, 0, C.byref(n))
        if rc not in (PA_OK, PA_ERR_ARG):
            _check(rc)
        out = np.zeros(max(1, n.value), dtype=np.int32)
        _check(self._lib.pa_seq_blocks(self._h, int(seq_id), _ptr(out), out.size, C.byref(n)))
        return out[:n.value].tolist()

    def free_list(self):
        n = C.c_int32(0)
        out = np.zeros(self.num_blocks, dtype=np.int32)
        _check(self._lib.pa_pool_free_list(self._h, _ptr(out), out.size, C.byref(n)))
        return out[:n.value].tolist()

    def metadata(self, seq_ids, q_lens, max_blocks_per_seq: int, out=None):
        """Block table, seq_lens, cu_seqlens_q and slot_mapping (numpy int32).
        ``out`` may supply preallocated arrays (e.g. pinned) to fill."""
        ids = np.ascontiguousarray(seq_ids, dtype=np.int64)
        ql = _i32(q_lens)
        n = ids.size
        total = int(ql.sum()) if n else 0
        if out is None:
            out = {"block_table": np.empty((n, max_blocks_per_seq), np.int32),
                   "seq_lens": np.empty(n, np.int32), "cu_seqlens_q": np.empty(n + 1, np.int32),
                   "slot_mapping": np.empty(total, np.int32)}
        bt, sl, cu, sm = (out["block_table"], out["seq_lens"], out["cu_seqlens_q"],
                          out["slot_mapping"])
        _check(self._lib.pa_build_metadata(
            self._h, n, ids.ctypes.data_as(_I64P) if n else None, _ptr(ql) if n else None,
            int(max_blocks_per_seq), _ptr(bt) if n else None, _ptr(sl) if n else None, _ptr(cu),
            _ptr(sm) if sm.size else None, sm.size))
        return out


def form_batches(adapter_ids, prompt_lens, bucket_bounds):
    """pa_form_batches: returns (order, position, batches) where batches is a
    list of (adapter, bucket, original indices)."""
    a, ln, bb = _i32(adapter_ids), _i32(prompt_lens), _i32(bucket_bounds)
    n = a.size
    if ln.size != n:
        raise ValueError("adapter_ids and prompt_lens differ in length")
    order, position = np.zeros(max(n, 1), np.int32), np.zeros(max(n, 1), np.int32)
    offs = np.zeros(n + 1, np.int32)
    badp, bbuck = np.zeros(max(n, 1), np.int32), np.zeros(max(n, 1), np.int32)
    nb = C.c_int32(0)
    _check(lib().pa_form_batches(n, _ptr(a) if n else None, _ptr(ln) if n else None, bb.size,
                                 _ptr(bb) if bb.size else None, _ptr(order), _ptr(position),
                                 _ptr(offs), _ptr(badp), _ptr(bbuck), C.byref(nb)))
    batches = [(int(badp[b]), int(bbuck[b]), order[offs[b]:offs[b + 1]].tolist())
               for b in range(nb.value)]
    return order[:n].tolist(), position[:n].tolist(), batches


def plan(kind: int, n_q: int, seq_lens, cu_seqlens_q, num_q_heads: int, num_kv_heads: int,
         head_dim: int, block_size: int, dtype: int, num_cus: int = 0, out=None,
         block_table=None):
    """Build the launch plan on the host; returns (int32 plan array, PlanInfo).
    ``out`` (int32 array, e.g. a pinned staging view) is used when large
    enough.  ``block_table`` (host [n_seqs, max_blocks] int32) enables
    shared-prefix groups."""
    L = lib()
    sl, cu = _i32(seq_lens), _i32(cu_seqlens_q)
    n = sl.size
    info = PlanInfo()
    if block_table is not None and n:
        bt = _i32(block_table)
        bt_ptr, mb = _ptr(bt), int(bt.shape[1])
    else:
        bt_ptr, mb = None, 0
    args = (int(kind), int(n_q), n, _ptr(sl) if n else None, _ptr(cu), bt_ptr, mb,
            int(num_q_heads), int(num_kv_heads), int(head_dim), int(block_size), int(dtype),
            int(num_cus))
    if out is not None:
        rc = L.pa_attn_plan(*args, _ptr(out), out.size, C.byref(info))
        if rc == PA_OK:
            return out[:info.plan_words], info
        if not (rc == PA_ERR_ARG and info.plan_words > out.size):
            _check(rc)
    else:
        _check(L.pa_attn_plan(*args, None, 0, C.byref(info)))
    arr = np.zeros(max(1, info.plan_words), dtype=np.int32)
    _check(L.pa_attn_plan(*args, _ptr(arr), arr.size, C.byref(info)))
    return arr[:info.plan_words], info


def workspace_size(total_q: int, num_q_heads: int, head_dim: int, max_seq_len: int,
                   decode: bool = False) -> int:
    """Bound on the split-K workspace of any plan for such a launch
    (pa_attn_workspace_size, or pa_attn_decode_workspace_size with total_q
    the number of decode sequences)."""
    n = C.c_size_t(0)
    fn = lib().pa_attn_decode_workspace_size if decode else lib().pa_attn_workspace_size
    _check(fn(int(total_q), int(num_q_heads), int(head_dim), int(max_seq_len), C.byref(n)))
    return int(n.value)


# Marshalling of the device calls.  In a layer of few requests the two calls'
# host time is what the GPU waits for (kv_append and attention of 4 short float32
# requests: 17.8 us on the host, 11 us of kernels), and half of it was these
# helpers: a Stream object made per call to read its handle (2.6 us; the handle
# itself 0.3 us), `import torch` and a table of entry points on every call.
def _dptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _torch_module():
    global _torch
    if _torch is None:
        import torch
        _torch = torch
        _ROW_DTYPES.update({torch.bfloat16: PA_BF16, torch.float32: PA_F32})
    return _torch


def _stream(stream) -> int:
    if stream is None:
        t = _torch or _torch_module()
        return t._C._cuda_getCurrentRawStream(t.cuda.current_device())
    return int(getattr(stream, "cuda_stream", stream))


_hip = None
HIP_EVENT_DISABLE_TIMING, HIP_EVENT_DISABLE_SYSTEM_FENCE = 0x2, 0x20000000


def _hip_runtime():
    """The HIP runtime libpa links against (the process's only copy: torch
    loads the same soname)."""
    global _hip
    if _hip is None:
        lib()
        h = C.CDLL("libamdhip64.so.7")
        h.hipEventCreateWithFlags.argtypes = [C.POINTER(_P), C.c_uint]
        h.hipEventRecord.argtypes = [_P, _P]
        h.hipEventSynchronize.argtypes = [_P]
        h.hipEventElapsedTime.argtypes = [C.POINTER(C.c_float), _P, _P]
        h.hipEventDestroy.argtypes = [_P]
        for f in ("hipEventCreateWithFlags", "hipEventRecord", "hipEventSynchronize",
                  "hipEventElapsedTime", "hipEventDestroy"):
            getattr(h, f).restype = C.c_int
        _hip = h
    return _hip


class StreamEvent:
    """A HIP event recorded without a system-scope fence.

    A default event record writes back and invalidates the GPU caches at
    system scope so the host can read device results once the event
    completes; in a stream of back-to-back kernels each such record costs
    several microseconds of idle device.  Nothing waiting on these events
    reads device memory: the staging buffers use them to learn that an
    upload has finished reading pinned host memory (its loads bypass the
    caches), and the benchmark uses them for timing only."""

    def __init__(self, timing: bool = False):
        self._h = _hip_runtime()
        self._ev = _P()
        flags = HIP_EVENT_DISABLE_SYSTEM_FENCE | (0 if timing else HIP_EVENT_DISABLE_TIMING)
        self._rc("hipEventCreateWithFlags", self._h.hipEventCreateWithFlags(C.byref(self._ev), flags))

    @staticmethod
    def _rc(what: str, rc: int):
        if rc != 0:
            raise PaError(PA_ERR_LAUNCH, f"{what} returned HIP error {rc}")

    def record(self, stream=None):
        self._rc("hipEventRecord", self._h.hipEventRecord(self._ev, _stream(stream)))

    def synchronize(self):
        self._rc("hipEventSynchronize", self._h.hipEventSynchronize(self._ev))

    def elapsed_time(self, end: "StreamEvent") -> float:
        """Milliseconds from this event to end (both recorded and complete)."""
        ms = C.c_float()
        self._rc("hipEventElapsedTime", self._h.hipEventElapsedTime(C.byref(ms), self._ev, end._ev))
        return float(ms.value)

    def __del__(self):
        if getattr(self, "_ev", None) and _hip is not None:
            _hip.hipEventDestroy(self._ev)
            self._ev = None


# Per-device workspace held by pa_attn_decode_noalloc (PA_NOALLOC_WORKSPACE_BYTES).
NOALLOC_WORKSPACE_BYTES = 32 << 20


def _dtype_code(t) -> int:
    torch = _torch or _torch_module()
    dt = t.dtype
    if dt == torch.bfloat16:
        return PA_BF16
    if dt == torch.float32:
        return PA_F32
    raise PaError(PA_ERR_UNSUPPORTED, f"dtype {dt}")


def stage_upload(dst, src, nbytes: int, stream=None):
    """Copy the first nbytes of pinned host tensor src into device tensor dst
    with the library's upload kernel (pa_stage_upload)."""
    _check(lib().pa_stage_upload(_dptr(dst), _dptr(src), int(nbytes), _stream(stream)))


def cache_dims(k_cache, v_cache):
    """(num_blocks, num_kv_heads, head_dim, block_size) of a paged cache: the
    value cache is [NB, Hkv, D, bs]; the key cache holds as many elements in
    the grouped layout [NB, Hkv, D / 32, bs, 32]."""
    nb, hkv, d, bs = v_cache.shape
    if k_cache.numel() != v_cache.numel() or k_cache.dtype != v_cache.dtype:
        raise PaError(PA_ERR_ARG, "key and value caches differ in size or dtype")
    return nb, hkv, d, bs


def kv_append(k_new, v_new, slot_mapping, k_cache, v_cache, stream=None):
    """Scatter new K/V ([T, Hkv, D] device tensors) into the paged cache."""
    nb, hkv, d, bs = cache_dims(k_cache, v_cache)
    _check((_lib or lib()).pa_kv_append(_dptr(k_new), _dptr(v_new), _dptr(slot_mapping),
                                        slot_mapping.numel(), _dptr(k_cache), _dptr(v_cache), nb,
                                        hkv, d, bs, _dtype_code(k_cache), _stream(stream)))


def attention(kind: int, q, k_cache, v_cache, block_table, seq_lens, cu_seqlens_q, plan_dev,
              info: PlanInfo, workspace, out, lse=None, scale=None, stream=None):
    """Paged attention (prefill / decode / verify by ``kind``) on device tensors."""
    nb, hkv, d, bs = cache_dims(k_cache, v_cache)
    total_q, hq, _ = q.shape
    if scale is None:
        scale = d ** -0.5
    if _lib is None:
        lib()
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(_attn[kind](_dptr(q), _dptr(k_cache), _dptr(v_cache), nb, _dptr(block_table),
                       block_table.shape[1], _dptr(seq_lens), _dptr(cu_seqlens_q),
                       seq_lens.numel(), total_q, hq, hkv, d, bs, float(scale), _dtype_code(q),
                       _dptr(plan_dev), C.byref(info), _dptr(workspace), ws_bytes, _dptr(out),
                       _dptr(lse), _stream(stream)))


def set_launch_events(start: "StreamEvent | None", stop: "StreamEvent | None"):
    """The next attention call on this thread records start when its first
    kernel starts and stop when its last kernel ends (events carried by the
    kernel dispatches, no event packets between kernels)."""
    _check(lib().pa_set_launch_events(start._ev if start is not None else None,
                                      stop._ev if stop is not None else None))


def attention_decode_noalloc(q, k_cache, v_cache, block_table, seq_lens, cu_seqlens_q, plan_dev,
                             info: PlanInfo, out, lse=None, scale=None, stream=None):
    """Decode through pa_attn_decode_noalloc (split-K partials in the
    library's per-device array; no workspace argument)."""
    nb, hkv, d, bs = cache_dims(k_cache, v_cache)
    total_q, hq, _ = q.shape
    if scale is None:
        scale = d ** -0.5
    _check((_lib or lib()).pa_attn_decode_noalloc(
        _dptr(q), _dptr(k_cache), _dptr(v_cache), nb, _dptr(block_table), block_table.shape[1],
        _dptr(seq_lens), _dptr(cu_seqlens_q), seq_lens.numel(), total_q, hq, hkv, d, bs,
        float(scale), _dtype_code(q), _dptr(plan_dev), C.byref(info), _dptr(out), _dptr(lse),
        _stream(stream)))


# -- the 8-bit and the 4-bit cache ---------------------------------------------
def kv8_cache_shapes(num_blocks: int, num_kv_heads: int, head_dim: int, block_size: int = 16):
    """Shapes of an 8-bit cache's (k_cache, v_cache, scales); the caches are
    torch.float8_e4m3fn, the scales torch.uint8 (exponent + 127 of keys and of
    values), in memory of a multiple of 4 bytes, as torch allocates it.  Contents need
    no initialisation."""
    return ((num_blocks, num_kv_heads, head_dim // 64, block_size, 64),
            (num_blocks, num_kv_heads, head_dim, block_size), (num_blocks, num_kv_heads, 2))


def kv4_cache_shapes(num_blocks: int, num_kv_heads: int, head_dim: int, block_size: int = 16):
    """Shapes of a 4-bit cache's (k_cache, v_cache, scales), all torch.uint8: two e2m1
    codes a byte; exponent + 127 for 32 dims of each token's key, and in the last row of
    its value.  Contents need no initialisation."""
    return ((num_blocks, num_kv_heads, block_size, head_dim // 2),
            (num_blocks, num_kv_heads, head_dim // 32, 16, block_size),
            (num_blocks, num_kv_heads, head_dim // 32 + 1, block_size))


# The calls below check every tensor they take (types, shapes, strides, device): a
# kernel given the wrong one reads past its buffers.  The checks are one expression
# of attribute reads; what is wrong is looked for only when it fails, as a call of
# few rows waits for the host (an append's checks and marshalling 9.5 us written
# plainly, 5 so, where the kernel takes 4).
def _refuse(code: int, checks):
    """Raise for the first (holds, message) that does not hold."""
    for holds, msg in checks:
        if not holds:
            raise PaError(code, msg)


def _refuse_cache(t, bits, dt, whole, k_cache, v_cache, scales):
    _refuse(PA_ERR_UNSUPPORTED, [(
        k_cache.dtype == v_cache.dtype == dt and scales.dtype == t.uint8,
        f"{bits}-bit cache of {k_cache.dtype}, {v_cache.dtype} and {scales.dtype} (supported: "
        f"{str(dt)[6:]} with uint8 scales)")])
    _refuse(PA_ERR_ARG, [
        (whole, f"{bits}-bit cache: k_cache, v_cache and scales differ in shape"),
        (k_cache.is_contiguous() and v_cache.is_contiguous() and scales.is_contiguous(),
         f"{bits}-bit cache: tensors must be contiguous")])


def _refuse_metadata(t, block_table, seq_lens, cu_seqlens):
    n = seq_lens.numel()
    _refuse(PA_ERR_ARG, [
        (block_table.dim() == 2 and block_table.shape[0] >= n and cu_seqlens.numel() > n,
         f"metadata of {n} sequences: block_table {tuple(block_table.shape)}, cu_seqlens "
         f"{cu_seqlens.numel()}"),
        (all(m.dtype == t.int32 and m.is_contiguous()
             for m in (block_table, seq_lens, cu_seqlens)),
         "metadata must be contiguous int32")])


def _refuse_device(*tensors):
    t = _torch or _torch_module()
    now = t.cuda.current_device() if t.cuda.is_available() else None
    for x in tensors:
        if x is not None and x.get_device() != now:
            raise PaError(PA_ERR_ARG, f"tensor on {x.device}: all tensors must be on the current "
                          f"GPU ({now})")


def _stream_on(device: int, stream) -> int:
    """The stream's handle, or the current one's; -1 where the current device is
    not ``device``."""
    c = _torch._C
    if device < 0 or c._cuda_getDevice() != device:
        return -1
    if stream is None:
        return c._cuda_getCurrentRawStream(device)
    return int(getattr(stream, "cuda_stream", stream))


def _packed(x, heads: int, d: int) -> bool:
    """Whether each row's heads of x [T, heads, d] lie side by side (in a column
    slice of a larger matrix they do)."""
    s = x.stride()
    return s[2] == 1 and (s[1] == d or heads == 1) or x.numel() == 0


def _quant_rows(fn, bits, k, v, block_table, seq_lens, cu_seqlens, k_cache, v_cache, scales, stream):
    # a call of few rows waits for these lines: each is asked for once, and written out
    t = _torch or _torch_module()
    i32, u8, vc = t.int32, t.uint8, v_cache.shape
    if bits == 8:
        cdt, (nb, hkv, d, bs) = t.float8_e4m3fn, vc
        whole = k_cache.shape == (nb, hkv, d // 64, bs, 64) and scales.shape == (nb, hkv, 2)
    elif len(vc) == 5:
        cdt, (nb, hkv, c, i, bs) = u8, vc
        d = 32 * c
        whole = (i == 16 and bs == 16 and scales.shape == (nb, hkv, c + 1, 16)
                 and k_cache.shape == (nb, hkv, 16, 16 * c))
    else:
        cdt, nb, hkv, d, bs, whole = u8, 0, 0, 0, 16, False
    shape, dt, n, ks, vs = k.shape, k.dtype, seq_lens.numel(), k.stride(), v.stride()
    T, code = shape[0], _ROW_DTYPES.get(dt)
    table = block_table.shape
    rows, width = table if len(table) == 2 else (-1, 0)
    dev = v_cache.get_device()
    st = _stream_on(dev, stream)
    # a row's heads packed: the last stride one, the heads' the width or of one head
    if not (shape == (T, hkv, d) and v.shape == shape
            and (ks[2] == vs[2] == 1 and (ks[1] == vs[1] == d or hkv == 1) or T == 0 or d == 0)
            and code is not None and v.dtype == dt
            and k_cache.dtype == cdt and v_cache.dtype == cdt and scales.dtype == u8 and whole
            and k_cache.is_contiguous() and v_cache.is_contiguous() and scales.is_contiguous()
            and rows >= n and cu_seqlens.numel() > n
            and block_table.dtype == i32 and seq_lens.dtype == i32 and cu_seqlens.dtype == i32
            and block_table.is_contiguous() and seq_lens.is_contiguous()
            and cu_seqlens.is_contiguous()
            and st >= 0 and k.get_device() == v.get_device() == k_cache.get_device()
            == scales.get_device() == block_table.get_device() == seq_lens.get_device()
            == cu_seqlens.get_device() == dev):
        _refuse_cache(t, bits, cdt, whole, k_cache, v_cache, scales)
        _refuse(PA_ERR_ARG, [
            (shape == (T, hkv, d) and v.shape == shape and _packed(k, hkv, d)
             and _packed(v, hkv, d),
             f"rows {tuple(k.shape)} of strides {k.stride()} and {tuple(v.shape)} of "
             f"{v.stride()}, expected [T, {hkv}, {d}] with a row's heads packed"),
            (dt == v.dtype, "keys and values differ in dtype")])
        _refuse_metadata(t, block_table, seq_lens, cu_seqlens)
        _dtype_code(k)
        _refuse_device(k, v, k_cache, v_cache, scales, block_table, seq_lens, cu_seqlens)
    # a single row's stride means nothing
    k_row, v_row = (ks[0], vs[0]) if T > 1 else (hkv * d, hkv * d)
    rc = fn(k.data_ptr(), k_row, v.data_ptr(), v_row, block_table.data_ptr(), width,
            seq_lens.data_ptr(), cu_seqlens.data_ptr(), n, T, k_cache.data_ptr(),
            v_cache.data_ptr(), scales.data_ptr(), nb, hkv, d, bs, code, st)
    if rc:
        _check(rc)


def kv8_append(k_new, v_new, block_table, seq_lens, cu_seqlens, k_cache, v_cache, scales,
               stream=None):
    """Quantise new K/V ([T, Hkv, D] device tensors, rows at any stride) into
    the 8-bit cache: rows cu_seqlens[r] .. cu_seqlens[r + 1] are sequence r's
    last positions."""
    _quant_rows((_lib or lib()).pa_kv8_append, 8, k_new, v_new, block_table, seq_lens, cu_seqlens,
                k_cache, v_cache, scales, stream)


def kv8_read(k_out, v_out, block_table, seq_lens, cu_seqlens, k_cache, v_cache, scales,
             stream=None):
    """Read tokens of the 8-bit cache into k_out and v_out ([T, Hkv, D]); rows
    as kv8_append's."""
    _quant_rows((_lib or lib()).pa_kv8_read, 8, k_out, v_out, block_table, seq_lens, cu_seqlens,
                k_cache, v_cache, scales, stream)


def kv4_append(k_new, v_new, block_table, seq_lens, cu_seqlens, k_cache, v_cache, scales,
               stream=None):
    """Quantise new K/V into the 4-bit cache; rows as kv8_append's."""
    _quant_rows((_lib or lib()).pa_kv4_append, 4, k_new, v_new, block_table, seq_lens, cu_seqlens,
                k_cache, v_cache, scales, stream)


def kv4_read(k_out, v_out, block_table, seq_lens, cu_seqlens, k_cache, v_cache, scales,
             stream=None):
    """Read tokens of the 4-bit cache into k_out and v_out; rows as kv8_append's."""
    _quant_rows((_lib or lib()).pa_kv4_read, 4, k_out, v_out, block_table, seq_lens, cu_seqlens,
                k_cache, v_cache, scales, stream)


def _quant_attn_args(bits, q, k_cache, v_cache, scales, block_table, seq_lens, cu_seqlens_q, plan_dev,
                     info, out, lse, scale, stream, workspace):
    """(arguments up to the plan info, stream) of a call over the 8- or 4-bit cache."""
    t = _torch or _torch_module()
    i32, bf16, u8, vc, shape = t.int32, t.bfloat16, t.uint8, v_cache.shape, q.shape
    if bits == 8:
        cdt, (nb, hkv, d, bs) = t.float8_e4m3fn, vc
        whole = k_cache.shape == (nb, hkv, d // 64, bs, 64) and scales.shape == (nb, hkv, 2)
    elif len(vc) == 5:
        cdt, (nb, hkv, c, i, bs) = u8, vc
        d = 32 * c
        whole = (i == 16 and bs == 16 and scales.shape == (nb, hkv, c + 1, 16)
                 and k_cache.shape == (nb, hkv, 16, 16 * c))
    else:
        cdt, nb, hkv, d, bs, whole = u8, 0, 0, 0, 16, False
    total_q, hq, dq = shape
    n, table = seq_lens.numel(), block_table.shape
    rows, width = table if len(table) == 2 else (-1, 0)
    dev = v_cache.get_device()
    st = _stream_on(dev, stream)
    if not (q.dtype == bf16 and out.dtype == bf16 and dq == d
            and out.shape == shape and q.is_contiguous() and out.is_contiguous()
            and k_cache.dtype == cdt and v_cache.dtype == cdt and scales.dtype == u8 and whole
            and k_cache.is_contiguous() and v_cache.is_contiguous() and scales.is_contiguous()
            and rows >= n and cu_seqlens_q.numel() > n
            and block_table.dtype == i32 and seq_lens.dtype == i32 and cu_seqlens_q.dtype == i32
            and block_table.is_contiguous() and seq_lens.is_contiguous()
            and cu_seqlens_q.is_contiguous()
            and (plan_dev is None or (plan_dev.dtype == i32 and plan_dev.is_contiguous()
                                      and plan_dev.numel() >= info.plan_words
                                      and plan_dev.get_device() == dev))
            and (lse is None or (lse.dtype == t.float32 and lse.shape == (total_q, hq)
                                 and lse.is_contiguous() and lse.get_device() == dev))
            and (workspace is None or (workspace.is_contiguous()
                                       and workspace.get_device() == dev))
            and st >= 0 and q.get_device() == out.get_device() == k_cache.get_device()
            == scales.get_device() == block_table.get_device() == seq_lens.get_device()
            == cu_seqlens_q.get_device() == dev):
        _refuse_cache(t, bits, cdt, whole, k_cache, v_cache, scales)
        _refuse(PA_ERR_UNSUPPORTED, [
            (q.dtype == out.dtype == t.bfloat16,
             f"queries {q.dtype}, output {out.dtype} (supported: bfloat16)")])
        _refuse(PA_ERR_ARG, [
            (dq == d and out.shape == q.shape and q.is_contiguous() and out.is_contiguous(),
             "q and out must be contiguous [T, Hq, D] of the cache's head_dim"),
            (lse is None or (lse.dtype == t.float32 and lse.shape == (total_q, hq)
                             and lse.is_contiguous()), "lse must be contiguous float32 [T, Hq]"),
            (plan_dev is None or (plan_dev.dtype == i32 and plan_dev.is_contiguous()
                                  and plan_dev.numel() >= info.plan_words),
             f"plan: contiguous int32 of at least its info's {info.plan_words} words"),
            (workspace is None or workspace.is_contiguous(), "workspace must be contiguous")])
        _refuse_metadata(t, block_table, seq_lens, cu_seqlens_q)
        _refuse_device(q, out, lse, k_cache, v_cache, scales, block_table, seq_lens, cu_seqlens_q,
                       plan_dev, workspace)
    return (q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), scales.data_ptr(), nb,
            block_table.data_ptr(), width, seq_lens.data_ptr(), cu_seqlens_q.data_ptr(), n,
            total_q, hq, hkv, d, bs, d ** -0.5 if scale is None else scale, _dptr(plan_dev),
            C.byref(info)), st


def kv8_attention(kind: int, q, k_cache, v_cache, scales, block_table, seq_lens, cu_seqlens_q,
                  plan_dev, info: PlanInfo, workspace, out, lse=None, scale=None, stream=None):
    """Paged attention over the 8-bit cache (prefill / decode / verify by
    ``kind``), with a plan built for PA_BF16_KV8."""
    if _lib is None:
        lib()
    args, st = _quant_attn_args(8, q, k_cache, v_cache, scales, block_table, seq_lens, cu_seqlens_q,
                                plan_dev, info, out, lse, scale, stream, workspace)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = _kv8_attn[kind](*args, _dptr(workspace), ws_bytes, out.data_ptr(), _dptr(lse), st)
    if rc:
        _check(rc)


def kv8_attention_decode_noalloc(q, k_cache, v_cache, scales, block_table, seq_lens, cu_seqlens_q,
                                 plan_dev, info: PlanInfo, out, lse=None, scale=None, stream=None):
    """Decode over the 8-bit cache with the split-K partials in the library's
    per-device array (as attention_decode_noalloc)."""
    fn = (_lib or lib()).pa_kv8_attn_decode_noalloc
    args, st = _quant_attn_args(8, q, k_cache, v_cache, scales, block_table, seq_lens, cu_seqlens_q,
                                plan_dev, info, out, lse, scale, stream, None)
    _check(fn(*args, out.data_ptr(), _dptr(lse), st))


def kv4_attention(kind: int, q, k_cache, v_cache, scales, block_table, seq_lens, cu_seqlens_q,
                  plan_dev, info: PlanInfo, workspace, out, lse=None, scale=None, stream=None):
    """Paged attention over the 4-bit cache (prefill / decode / verify by
    ``kind``), with a plan built for PA_BF16_KV4."""
    if _lib is None:
        lib()
    args, st = _quant_attn_args(4, q, k_cache, v_cache, scales, block_table, seq_lens, cu_seqlens_q,
                                plan_dev, info, out, lse, scale, stream, workspace)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = _kv4_attn[kind](*args, _dptr(workspace), ws_bytes, out.data_ptr(), _dptr(lse), st)
    if rc:
        _check(rc)


def kv4_attention_decode_noalloc(q, k_cache, v_cache, scales, block_table, seq_lens, cu_seqlens_q,
                                 plan_dev, info: PlanInfo, out, lse=None, scale=None, stream=None):
    """Decode over the 4-bit cache with the split-K partials in the library's
    per-device array (as attention_decode_noalloc)."""
    fn = (_lib or lib()).pa_kv4_attn_decode_noalloc
    args, st = _quant_attn_args(4, q, k_cache, v_cache, scales, block_table, seq_lens, cu_seqlens_q,
                                plan_dev, info, out, lse, scale, stream, None)
    _check(fn(*args, out.data_ptr(), _dptr(lse), st))


# -- eviction from live contexts ------------------------------------------------
def _plain_form(t, k_cache, scales):
    """(dtype code, blocks, kv-heads, head_dim, block size) of the cache that k_cache, and for
    the 4-bit cache scales, are part of; code None: no cache that the calls below take."""
    dt, dim = k_cache.dtype, k_cache.dim()
    if scales is not None:
        if dim != 4 or dt != t.uint8:
            return None, 0, 0, 0, 16
        nb, hkv, bs, half = k_cache.shape
        return PA_BF16_KV4, nb, hkv, 2 * half, bs
    code = _ROW_DTYPES.get(dt)
    if dim != 5 or k_cache.shape[4] != 32:
        return None, 0, 0, 0, 16
    nb, hkv, groups, bs, _ = k_cache.shape
    return code, nb, hkv, 32 * groups, bs


def attention_weights(q, lse, k_cache, block_table, seq_lens, cu_seqlens_q, weights, scales=None,
                      accumulate: bool = False, scale=None, stream=None):
    """weights[r, h, t] (float32 [n_seqs, Hkv, >= longest sequence]): the probabilities of
    cached key t summed over the rows of sequence r and the query heads of kv-head h, from
    an attention call's queries and log-sum-exps; added to what is there with
    ``accumulate``.  k_cache of a bf16 cache, or of a 4-bit one with its scales."""
    t = _torch or _torch_module()
    fn = (_lib or lib()).pa_attn_weights
    code, nb, hkv, d, bs = _plain_form(t, k_cache, scales)
    total_q, hq, dq = q.shape
    n, i32 = seq_lens.numel(), t.int32
    rows, width = block_table.shape if block_table.dim() == 2 else (-1, 0)
    dev = k_cache.get_device()
    st = _stream_on(dev, stream)
    if not (code in (PA_BF16, PA_BF16_KV4) and q.dtype == t.bfloat16 and dq == d
            and q.is_contiguous() and k_cache.is_contiguous()
            and lse.dtype == t.float32 and lse.shape == (total_q, hq) and lse.is_contiguous()
            and weights.dtype == t.float32 and weights.dim() == 3 and weights.shape[0] >= n
            and weights.shape[1] == hkv and weights.is_contiguous()
            and (scales is None or (scales.dtype == t.uint8 and scales.is_contiguous()
                 and scales.shape == (nb, hkv, d // 32 + 1, 16) and scales.get_device() == dev))
            and rows >= n and cu_seqlens_q.numel() > n
            and block_table.dtype == i32 and seq_lens.dtype == i32 and cu_seqlens_q.dtype == i32
            and block_table.is_contiguous() and seq_lens.is_contiguous()
            and cu_seqlens_q.is_contiguous()
            and st >= 0 and q.get_device() == lse.get_device() == weights.get_device()
            == block_table.get_device() == seq_lens.get_device() == cu_seqlens_q.get_device() == dev):
        _refuse(PA_ERR_UNSUPPORTED, [
            (code in (PA_BF16, PA_BF16_KV4), f"keys {k_cache.dtype} {tuple(k_cache.shape)}"
             f"{'' if scales is None else ' with scales'}: supported are a bf16 cache's, or a "
             "4-bit cache's with its scales"),
            (q.dtype == t.bfloat16, f"queries {q.dtype} (supported: bfloat16)")])
        _refuse(PA_ERR_ARG, [
            (dq == d and q.is_contiguous(), "q must be contiguous [T, Hq, D] of the cache's head_dim"),
            (k_cache.is_contiguous(), "k_cache must be contiguous"),
            (lse.dtype == t.float32 and lse.shape == (total_q, hq) and lse.is_contiguous(),
             "lse must be contiguous float32 [T, Hq]"),
            (weights.dtype == t.float32 and weights.dim() == 3 and weights.shape[0] >= n
             and weights.shape[1] == hkv and weights.is_contiguous(),
             f"weights must be contiguous float32 [{n}, {hkv}, keys]"),
            (scales is None or (scales.dtype == t.uint8 and scales.is_contiguous()
             and scales.shape == (nb, hkv, d // 32 + 1, 16)),
             f"scales must be contiguous uint8 [{nb}, {hkv}, {d // 32 + 1}, 16]")])
        _refuse_metadata(t, block_table, seq_lens, cu_seqlens_q)
        _refuse_device(q, lse, k_cache, scales, weights, block_table, seq_lens, cu_seqlens_q)
    rc = fn(q.data_ptr(), lse.data_ptr(), k_cache.data_ptr(), _dptr(scales), nb,
            block_table.data_ptr(), width, seq_lens.data_ptr(), cu_seqlens_q.data_ptr(), n, total_q,
            hq, hkv, d, bs, d ** -0.5 if scale is None else scale, code, weights.data_ptr(),
            weights.shape[2], int(bool(accumulate)), st)
    if rc:
        _check(rc)


def kv_evict(weights, block_table, seq_lens, new_lens, k_cache, v_cache, kept, scales=None,
             new_table=None, weights_out=None, first=None, window: int = 0, stream=None):
    """Shorten sequences to new_lens tokens: the first ``first[r]``, the last ``window`` and
    the heaviest of the rest stay, for each kv-head its own.  kept (int32 [n_seqs, Hkv, >=
    longest new length]) receives their positions, weights_out (default: weights itself)
    their weights; keys and values move to the blocks of new_table, by default within the
    sequence's own.  A float32, bf16 or, with its scales, 4-bit cache."""
    t = _torch or _torch_module()
    fn = (_lib or lib()).pa_kv_evict
    code, nb, hkv, d, bs = _plain_form(t, k_cache, scales)
    v_shape = (nb, hkv, d // 32, 16, 16) if scales is not None else (nb, hkv, d, bs)
    n, i32, f32 = seq_lens.numel(), t.int32, t.float32
    if weights_out is None:
        weights_out = weights
    dev = k_cache.get_device()
    st = _stream_on(dev, stream)
    lists = (seq_lens, new_lens) if first is None else (seq_lens, new_lens, first)
    tables = (block_table,) if new_table is None else (block_table, new_table)

    def spare(x, dtype):
        return (x.dtype == dtype and x.dim() == 3 and x.shape[0] >= n and x.shape[1] == hkv
                and x.is_contiguous())

    if not (code is not None and v_cache.dtype == k_cache.dtype and v_cache.shape == v_shape
            and k_cache.is_contiguous() and v_cache.is_contiguous()
            and (scales is None or (scales.dtype == t.uint8 and scales.is_contiguous()
                 and scales.shape == (nb, hkv, d // 32 + 1, 16) and scales.get_device() == dev))
            and spare(weights, f32) and spare(weights_out, f32)
            and weights_out.shape[2] == weights.shape[2] and spare(kept, i32)
            and all(x.dtype == i32 and x.numel() == n and x.is_contiguous()
                    and x.get_device() == dev for x in lists)
            and all(x.dtype == i32 and x.dim() == 2 and x.shape[0] >= n and x.is_contiguous()
                    and x.get_device() == dev and (x.shape[1] > 0 or n == 0) for x in tables)
            and st >= 0 and v_cache.get_device() == weights.get_device()
            == weights_out.get_device() == kept.get_device() == dev):
        _refuse(PA_ERR_UNSUPPORTED, [
            (code is not None, f"keys {k_cache.dtype} {tuple(k_cache.shape)}"
             f"{'' if scales is None else ' with scales'}: supported are a float32 or bf16 "
             "cache's, or a 4-bit cache's with its scales")])
        _refuse(PA_ERR_ARG, [
            (v_cache.dtype == k_cache.dtype and v_cache.shape == v_shape
             and k_cache.is_contiguous() and v_cache.is_contiguous(),
             f"k_cache and v_cache must be contiguous, v_cache {v_shape} of k_cache's type"),
            (scales is None or (scales.dtype == t.uint8 and scales.is_contiguous()
             and scales.shape == (nb, hkv, d // 32 + 1, 16)),
             f"scales must be contiguous uint8 [{nb}, {hkv}, {d // 32 + 1}, 16]"),
            (spare(weights, f32) and spare(weights_out, f32)
             and weights_out.shape[2] == weights.shape[2],
             f"weights and weights_out must be contiguous float32 [{n}, {hkv}, keys] of one width"),
            (spare(kept, i32), f"kept must be contiguous int32 [{n}, {hkv}, longest new length]"),
            (all(x.dtype == i32 and x.numel() == n and x.is_contiguous() for x in lists),
             f"seq_lens, new_lens and first must be contiguous int32 of {n} sequences"),
            # a table of no blocks has no address, which would mean a move in place
            (all(x.dtype == i32 and x.dim() == 2 and x.shape[0] >= n and x.is_contiguous()
                 and (x.shape[1] > 0 or n == 0) for x in tables),
             f"tables must be contiguous int32 [{n}, 1 block or more]")])
        _refuse_device(k_cache, v_cache, scales, weights, weights_out, kept, *lists, *tables)
    rc = fn(weights.data_ptr(), weights_out.data_ptr(), weights.shape[2], block_table.data_ptr(),
            block_table.shape[1], _dptr(new_table), 0 if new_table is None else new_table.shape[1],
            seq_lens.data_ptr(), new_lens.data_ptr(), _dptr(first), int(window), n,
            k_cache.data_ptr(), v_cache.data_ptr(), _dptr(scales), nb, hkv, d, bs, code,
            kept.data_ptr(), kept.shape[2], st)
    if rc:
        _check(rc)


def qk_norm_rope(q, k, positions, cos_sin, q_out, k_out, q_weight=None, k_weight=None,
                 eps: float = 1e-6, norm: bool = True, interleaved: bool = False, stream=None):
    """Normalise (``norm``) and rotate queries [T, Hq, D] and keys [T, Hkv, D]
    (rows at any stride) by their int32 positions and the float32 table cos_sin
    [n_positions, rot_dim] (cosines, then sines), into packed q_out and k_out."""
    t = _torch or _torch_module()
    fn = (_lib or lib()).pa_qk_norm_rope
    T, hq, d = q.shape
    hkv = k.shape[1]
    dt, dev = q.dtype, q_out.get_device()
    st, code = _stream_on(dev, stream), _ROW_DTYPES.get(dt)
    n_pos, rot = cos_sin.shape if cos_sin.dim() == 2 else (-1, 0)
    if not (k.shape == (T, hkv, d) and _packed(q, hq, d) and _packed(k, hkv, d)
            and code is not None and k.dtype == dt
            and q_out.dtype == dt and q_out.shape == (T, hq, d) and q_out.is_contiguous()
            and k_out.dtype == dt and k_out.shape == (T, hkv, d) and k_out.is_contiguous()
            and positions.dtype == t.int32 and positions.numel() == T
            and positions.is_contiguous() and n_pos >= 0 and cos_sin.dtype == t.float32
            and cos_sin.is_contiguous()
            and (q_weight is None or (q_weight.dtype == dt and q_weight.numel() == d
                 and q_weight.is_contiguous() and q_weight.get_device() == dev))
            and (k_weight is None or (k_weight.dtype == dt and k_weight.numel() == d
                 and k_weight.is_contiguous() and k_weight.get_device() == dev))
            and st >= 0 and q.get_device() == k.get_device() == k_out.get_device()
            == positions.get_device() == cos_sin.get_device() == dev):
        _refuse(PA_ERR_ARG, [
            (k.shape == (T, hkv, d) and _packed(q, hq, d) and _packed(k, hkv, d),
             f"q {tuple(q.shape)} of strides {q.stride()} and k {tuple(k.shape)} of "
             f"{k.stride()}: expected [T, Hq, D] and [T, Hkv, D] with a row's heads packed"),
            (k.dtype == dt, "q and k differ in dtype")]
            + [(x.shape == (T, h, d) and x.is_contiguous() and x.dtype == dt,
                f"{what} must be contiguous [{T}, {h}, {d}] of q's dtype")
               for x, h, what in ((q_out, hq, "q_out"), (k_out, hkv, "k_out"))]
            + [(w is None or (w.numel() == d and w.dtype == dt and w.is_contiguous()),
                f"{what} must be {d} contiguous values of q's dtype")
               for w, what in ((q_weight, "q_weight"), (k_weight, "k_weight"))]
            + [(positions.numel() == T and positions.dtype == t.int32
                and positions.is_contiguous(), "one contiguous int32 position per token"),
               (n_pos >= 0 and cos_sin.dtype == t.float32 and cos_sin.is_contiguous(),
                "cos_sin must be contiguous float32 [n_positions, rot_dim]")])
        _dtype_code(q)
        _refuse_device(q, k, q_out, k_out, positions, cos_sin, q_weight, k_weight)
    qs, ks = (q.stride(0), k.stride(0)) if T > 1 else (hq * d, hkv * d)
    rc = fn(q.data_ptr(), qs, k.data_ptr(), ks, positions.data_ptr(), T, cos_sin.data_ptr(),
            n_pos, rot, _dptr(q_weight), _dptr(k_weight), eps,
            (QK_NORM if norm else 0) | (ROPE_INTERLEAVED if interleaved else 0),
            q_out.data_ptr(), k_out.data_ptr(), hq, hkv, d, code, st)
    if rc:
        _check(rc)
