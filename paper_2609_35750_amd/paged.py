"""Python binding of the streamed paged KV cache of libkvs (ctypes).

The inference side of KV-streams (Section 2, "KV-streams"; Section 4,
"Inference engine implementation"): one (K, V) entry per generated token in
a paged cache, evicted entries dropped in place, and decode attention over
the entries live when a query is generated.  ``PagedKVCache`` owns the device
pools (torch tensors: memory only) and a native block manager; every step
runs in libkvs (host bookkeeping in C++, updates and attention in HIP
kernels).  Argument marshalling only.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Sequence, Tuple

import numpy as np
import torch

from .kvs import KVS_ERR_UNSUPPORTED, KvsError, _check, _i31, _on, _ptr, _stream, _workspace, lib


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _np_ptr(a: np.ndarray):
    return a.__array_interface__["data"][0]


class BlockManager:
    """Host-side block bookkeeping (``kvs_bm_*``)."""

    def __init__(self, num_blocks: int, block_size: int, num_seqs: int, max_blocks: int):
        h = ctypes.c_void_p()
        _check("kvs_bm_create", lib.kvs_bm_create(num_blocks, block_size, num_seqs, max_blocks, ctypes.byref(h)))
        self._h = h
        self.num_blocks, self.block_size, self.num_seqs, self.max_blocks = num_blocks, block_size, num_seqs, max_blocks

    def __del__(self):
        h = getattr(self, "_h", None)
        if h is not None and h.value:
            lib.kvs_bm_destroy(h)
            self._h = None

    def append(self, seq: int, positions: Sequence[int]) -> np.ndarray:
        pos = _i32(positions)
        slots = np.empty_like(pos)
        _check("kvs_bm_append", lib.kvs_bm_append(self._h, seq, _np_ptr(pos), pos.size, _np_ptr(slots)))
        return slots

    def evict(self, seq: int, positions: Sequence[int]) -> np.ndarray:
        pos = _i32(positions)
        slots = np.empty_like(pos)
        _check("kvs_bm_evict", lib.kvs_bm_evict(self._h, seq, _np_ptr(pos), pos.size, _np_ptr(slots)))
        return slots

    def release(self, seq: int) -> np.ndarray:
        slots = np.empty(max(self.live(seq), 1), dtype=np.int32)
        n = ctypes.c_int()
        _check("kvs_bm_release", lib.kvs_bm_release(self._h, seq, _np_ptr(slots), ctypes.byref(n)))
        return slots[: n.value]

    def fork(self, src: int, dst: int) -> None:
        _check("kvs_bm_fork", lib.kvs_bm_fork(self._h, src, dst))

    def _pairs(self, seq: int):
        """Room for (source, destination) slots of a sequence's entries, and their number."""
        return np.empty((2, max(self.live(seq), 1)), dtype=np.int32), ctypes.c_int()

    def evict_shared(self, seq: int, positions: Sequence[int]) -> Tuple[np.ndarray, np.ndarray]:
        """(slots as ``evict`` gives them, -1 for entries in shared blocks; [2, n] slots to copy from and to)."""
        pos = _i32(positions)
        slots = np.empty_like(pos)
        pairs, n = self._pairs(seq)
        _check("kvs_bm_evict_shared", lib.kvs_bm_evict_shared(
            self._h, seq, _np_ptr(pos), pos.size, _np_ptr(slots), _np_ptr(pairs), _np_ptr(pairs[1]), ctypes.byref(n)))
        return slots, pairs[:, : n.value]

    def copy(self, src: int, dst: int) -> np.ndarray:
        """[2, n] slots to copy from and to."""
        pairs, n = self._pairs(src)
        _check("kvs_bm_copy", lib.kvs_bm_copy(self._h, src, dst, _np_ptr(pairs), _np_ptr(pairs[1]), ctypes.byref(n)))
        return pairs[:, : n.value]

    def compact(self, seq: int) -> np.ndarray:
        """[2, n] slots to move from and to."""
        pairs, n = self._pairs(seq)
        _check("kvs_bm_compact", lib.kvs_bm_compact(self._h, seq, _np_ptr(pairs), _np_ptr(pairs[1]), ctypes.byref(n)))
        return pairs[:, : n.value]

    def groups(self) -> Tuple[np.ndarray, np.ndarray]:
        """Group of every sequence (-1: none), leading blocks each group has in common."""
        group, blocks = np.empty((2, self.num_seqs), dtype=np.int32)
        n = ctypes.c_int()
        _check("kvs_bm_groups", lib.kvs_bm_groups(self._h, _np_ptr(group), _np_ptr(blocks), ctypes.byref(n)))
        return group, blocks[: n.value]

    def shared(self, seq: int) -> int:
        return lib.kvs_bm_shared(self._h, seq)

    def tables(self) -> Tuple[np.ndarray, np.ndarray]:
        table = np.empty((self.num_seqs, self.max_blocks), dtype=np.int32)
        nblk = np.empty(self.num_seqs, dtype=np.int32)
        _check("kvs_bm_tables", lib.kvs_bm_tables(self._h, _np_ptr(table), _np_ptr(nblk)))
        return table, nblk

    def free_blocks(self) -> int:
        return lib.kvs_bm_free_blocks(self._h)

    def live(self, seq: int) -> int:
        return lib.kvs_bm_live(self._h, seq)


def kvs_paged_append(k_new, v_new, positions, slots, k_cache, v_cache, slot_pos, block_size: int) -> None:
    """``kvs_paged_append``: k_new/v_new [n, Hkv, D] bf16, positions/slots int32 [n] (device)."""
    n, Hkv, D = k_new.shape
    nb = k_cache.shape[0]
    _check("kvs_paged_append", lib.kvs_paged_append(
        _ptr(k_new), _ptr(v_new), _ptr(positions), _ptr(slots), n, _ptr(k_cache), _ptr(v_cache), _ptr(slot_pos),
        nb, block_size, Hkv, D, _stream(k_cache)))


def kvs_paged_evict(slots, slot_pos, num_blocks: int, block_size: int) -> None:
    _check("kvs_paged_evict", lib.kvs_paged_evict(_ptr(slots), slots.numel(), _ptr(slot_pos), num_blocks,
                                                   block_size, _stream(slot_pos)))


def kvs_paged_decode(q, k_cache, v_cache, slot_pos, block_table, seq_blocks, softmax_scale=None,
                     out=None, lse=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``kvs_paged_decode``: q [S, Hq, D] bf16; caches [num_blocks, Hkv, block_size, D]; returns (O, LSE)."""
    S, Hq, D = q.shape
    nb, Hkv, bs, Dk = k_cache.shape
    if Dk != D or v_cache.shape != k_cache.shape:
        raise ValueError("cache shapes do not match q")
    if q.dtype != torch.bfloat16 or k_cache.dtype != torch.bfloat16 or v_cache.dtype != torch.bfloat16:
        raise ValueError("q and the caches must be bfloat16")
    for t in (slot_pos, block_table, seq_blocks):
        if t.dtype != torch.int32:
            raise ValueError("slot_pos, block_table and seq_blocks must be int32")
    if block_table.dim() != 2 or block_table.shape[0] != S or seq_blocks.shape != (S,):
        raise ValueError("block_table must be [S, max_blocks] and seq_blocks [S]")
    if slot_pos.numel() != nb * bs:
        raise ValueError("slot_pos must hold num_blocks * block_size entries")
    max_blocks = block_table.shape[1]
    scale = 1.0 / math.sqrt(D) if softmax_scale is None else float(softmax_scale)
    o = torch.empty_like(q) if out is None else out
    lse = torch.empty((S, Hq), dtype=torch.float32, device=q.device) if lse is None else lse
    need = lib.kvs_paged_decode_workspace(S, Hq, Hkv, D, max_blocks, bs)
    ws = _workspace(need, q.device)
    _check("kvs_paged_decode", lib.kvs_paged_decode(
        _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(slot_pos), _ptr(block_table), _ptr(seq_blocks), _ptr(o),
        _ptr(lse), S, Hq, Hkv, D, nb, bs, max_blocks, scale, _ptr(ws), need, _stream(q)))
    return o, lse


def _same_device(ref, *tensors) -> None:
    for t in tensors:
        if t is not None and t.device != ref.device:
            raise ValueError("tensors must be on one device")
    if not ref.is_cuda:
        raise ValueError("tensors must be on the GPU")


def _int32(*tensors) -> None:
    for t in tensors:
        if t.dtype != torch.int32:
            raise ValueError("positions, slots, tables and counts must be int32")


def kvs_paged_append_weighted(k_new, v_new, w_new, positions, slots, k_cache, v_cache, slot_pos, slot_weight,
                              block_size: int) -> None:
    """``kvs_paged_append_weighted``: as ``kvs_paged_append``, with the entries' weights w_new float32 [n] (None: 0)."""
    n, Hkv, D = k_new.shape
    nb = k_cache.shape[0]
    if v_new.shape != k_new.shape or positions.shape != (n,) or slots.shape != (n,):
        raise ValueError("k_new, v_new, positions and slots do not match")
    if k_cache.shape != (nb, Hkv, block_size, D) or v_cache.shape != k_cache.shape or slot_pos.numel() != nb * block_size:
        raise ValueError("the caches must be [num_blocks, Hkv, block_size, D] with k_new's Hkv and D, slot_pos one entry a slot")
    if any(t.dtype != torch.bfloat16 for t in (k_new, v_new, k_cache, v_cache)):
        raise ValueError("k_new, v_new and the caches must be bfloat16")
    if slot_weight.dtype != torch.float32 or slot_weight.numel() != nb * block_size:
        raise ValueError("slot_weight must be float32 with num_blocks * block_size entries")
    if w_new is not None and (w_new.dtype != torch.float32 or w_new.shape != (n,)):
        raise ValueError("w_new must be float32 [n]")
    _int32(positions, slots, slot_pos)
    _same_device(k_cache, k_new, v_new, w_new, positions, slots, v_cache, slot_pos, slot_weight)
    with _on(k_cache):
        _check("kvs_paged_append_weighted", lib.kvs_paged_append_weighted(
            _ptr(k_new), _ptr(v_new), _ptr(w_new), _ptr(positions), _ptr(slots), n, _ptr(k_cache), _ptr(v_cache),
            _ptr(slot_pos), _ptr(slot_weight), nb, block_size, Hkv, D, _stream(k_cache)))


def kvs_paged_decode_ex(q, k_cache, v_cache, slot_pos, block_table, seq_blocks, softmax_scale=None, q_pos=None,
                        window: Optional[int] = None, sinks: int = 0, slot_weight=None, out=None,
                        lse=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``kvs_paged_decode_ex``: ``kvs_paged_decode`` under a sliding window, and with the entries' weights.

    ``window`` (None: none) with ``q_pos`` int32 [S], the queries' trace positions: of the live entries those at
    p <= q_pos with ``q_pos - p < window or p < sinks`` are seen.  ``slot_weight`` float32 [num_blocks * block_size]
    is added to in place: the attention weight, over all q-heads, of every entry its sequence's query sees.
    """
    S, Hq, D = q.shape
    nb, Hkv, bs, Dk = k_cache.shape
    if Dk != D or v_cache.shape != k_cache.shape:
        raise ValueError("cache shapes do not match q")
    if q.dtype != torch.bfloat16 or k_cache.dtype != torch.bfloat16 or v_cache.dtype != torch.bfloat16:
        raise ValueError("q and the caches must be bfloat16")
    _int32(slot_pos, block_table, seq_blocks)
    if block_table.dim() != 2 or block_table.shape[0] != S or seq_blocks.shape != (S,):
        raise ValueError("block_table must be [S, max_blocks] and seq_blocks [S]")
    if slot_pos.numel() != nb * bs:
        raise ValueError("slot_pos must hold num_blocks * block_size entries")
    if window is not None:
        if window < 1:
            raise ValueError("window must be >= 1 (None: no window)")
        if q_pos is None:
            raise ValueError("a window needs the queries' positions q_pos")
        _int32(q_pos)
        if q_pos.shape != (S,):
            raise ValueError("q_pos must be [S]")
    else:
        q_pos = None
    if slot_weight is not None and (slot_weight.dtype != torch.float32 or slot_weight.numel() != nb * bs):
        raise ValueError("slot_weight must be float32 with num_blocks * block_size entries")
    if out is not None and (out.shape != q.shape or out.dtype != torch.bfloat16):
        raise ValueError("O must have q's shape and type")
    if lse is not None and (lse.shape != (S, Hq) or lse.dtype != torch.float32):
        raise ValueError("LSE must be float32 [S, Hq]")
    _same_device(q, k_cache, v_cache, slot_pos, block_table, seq_blocks, q_pos, slot_weight, out, lse)
    max_blocks = block_table.shape[1]
    scale = 1.0 / math.sqrt(D) if softmax_scale is None else float(softmax_scale)
    o = torch.empty_like(q) if out is None else out
    lse = torch.empty((S, Hq), dtype=torch.float32, device=q.device) if lse is None else lse
    win, sinks = _i31(window or 0), _i31(sinks)
    need = lib.kvs_paged_decode_ex_workspace(S, Hq, Hkv, D, nb, max_blocks, bs, win, sinks, slot_weight is not None)
    ws = _workspace(need, q.device)
    with _on(q):
        _check("kvs_paged_decode_ex", lib.kvs_paged_decode_ex(
            _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(slot_pos), _ptr(slot_weight), _ptr(block_table),
            _ptr(seq_blocks), _ptr(q_pos), _ptr(o), _ptr(lse), S, Hq, Hkv, D, nb, bs, max_blocks, scale, win, sinks,
            _ptr(ws), need, _stream(q)))
    return o, lse


def kvs_paged_evict_lowest(slot_weight, slot_pos, block_table, seq_blocks, keep, block_size: int, sinks: int = 0,
                           recent: int = 0, max_out: Optional[int] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``kvs_paged_evict_lowest``: evicts the entries of lowest weight until ``keep`` int32 [S] are left a sequence.

    Positions below ``sinks`` and the ``recent`` positions up to the newest stay.  Marks the slots in ``slot_pos``
    and returns the evicted positions int32 [S, max_out] (in the table's order, then -1; ``max_out`` None: the
    table's width) and their numbers int32 [S].  The block manager learns of them through ``evict``.
    """
    if block_table.dim() != 2 or seq_blocks.shape != (block_table.shape[0],) or keep.shape != seq_blocks.shape:
        raise ValueError("block_table must be [S, max_blocks], seq_blocks and keep [S]")
    _int32(slot_pos, block_table, seq_blocks, keep)
    if max_out is not None and max_out > 0x7FFFFFFF:
        raise ValueError("max_out must fit 32 bits")
    if block_size < 1 or slot_pos.numel() % block_size:
        raise ValueError("slot_pos must hold num_blocks * block_size entries")
    if slot_weight.dtype != torch.float32 or slot_weight.numel() != slot_pos.numel():
        raise ValueError("slot_weight must be float32 with num_blocks * block_size entries")
    _same_device(slot_pos, slot_weight, block_table, seq_blocks, keep)
    S, max_blocks = block_table.shape
    most = max_blocks * block_size if max_out is None else int(max_out)
    pos = torch.empty((S, max(most, 0)), dtype=torch.int32, device=slot_pos.device)
    counts = torch.empty(S, dtype=torch.int32, device=slot_pos.device)
    need = lib.kvs_paged_evict_lowest_workspace(S, max_blocks, block_size)
    ws = _workspace(need, slot_pos.device) if need else None
    with _on(slot_pos):
        _check("kvs_paged_evict_lowest", lib.kvs_paged_evict_lowest(
            _ptr(slot_weight), _ptr(slot_pos), _ptr(block_table), _ptr(seq_blocks), _ptr(keep), _ptr(pos), _ptr(counts),
            S, slot_pos.numel() // block_size, block_size, max_blocks, _i31(sinks), _i31(recent), most, _ptr(ws), need,
            _stream(slot_pos)))
    return pos, counts


def kvs_paged_copy(src, dst, k_cache, v_cache, slot_pos=None, slot_weight=None, move: bool = False) -> None:
    """``kvs_paged_copy``: slot ``dst[i]`` takes the entry of slot ``src[i]`` (int32 [n]); ``move`` empties the sources.

    With its position where ``slot_pos`` is given, and its weight where ``slot_weight`` is.
    """
    cache, n = k_cache.shape, src.shape
    if len(cache) != 4 or v_cache.shape != cache:
        raise ValueError("the caches must be [num_blocks, Hkv, block_size, D]")
    if not k_cache.dtype == v_cache.dtype == torch.bfloat16:
        raise ValueError("the caches must be bfloat16")
    nb, Hkv, bs, D = cache
    if slot_pos is not None and (slot_pos.dtype != torch.int32 or slot_pos.numel() != nb * bs):
        raise ValueError("slot_pos must be int32 with num_blocks * block_size entries")
    if slot_weight is not None and (slot_weight.dtype != torch.float32 or slot_weight.numel() != nb * bs):
        raise ValueError("slot_weight must be float32 with num_blocks * block_size entries")
    if not src.dtype == dst.dtype == torch.int32:
        raise ValueError("positions, slots, tables and counts must be int32")
    if len(n) != 1 or dst.shape != n:
        raise ValueError("src and dst must be [n]")
    dev = k_cache.get_device()
    for t in (v_cache, src, dst, slot_pos, slot_weight):
        if t is not None and t.get_device() != dev:
            raise ValueError("tensors must be on one device")
    if dev < 0:
        raise ValueError("tensors must be on the GPU")
    with _on(k_cache):
        _check("kvs_paged_copy", lib.kvs_paged_copy(
            _ptr(src), _ptr(dst), n[0], _ptr(k_cache), _ptr(v_cache), _ptr(slot_pos), _ptr(slot_weight), int(move),
            nb, bs, Hkv, D, _stream(k_cache)))


def _rows_args(q, k_cache, v_cache, slot_pos, block_table, seq_blocks, softmax_scale, out, lse, a, b):
    """Checks shared by the calls with many query rows (a, b: two int32 tensors of the call's own).

    Returns (n, Hq, D, num_blocks, Hkv, block_size, S, max_blocks, O, LSE, scale)."""
    shape, cache, table = q.shape, k_cache.shape, block_table.shape
    if len(cache) != 4 or v_cache.shape != cache:
        raise ValueError("the caches must be [num_blocks, Hkv, block_size, D]")
    if not k_cache.dtype == v_cache.dtype == torch.bfloat16:
        raise ValueError("the caches must be bfloat16")
    nb, Hkv, bs, D = cache
    if slot_pos.dtype != torch.int32 or slot_pos.numel() != nb * bs:
        raise ValueError("slot_pos must be int32 with num_blocks * block_size entries")
    if len(shape) != 3 or q.dtype != torch.bfloat16:
        raise ValueError("q must be bfloat16 [n, Hq, D]")
    n, Hq, Dq = shape
    if Dq != D:
        raise ValueError("cache shapes do not match q")
    if not block_table.dtype == seq_blocks.dtype == a.dtype == b.dtype == torch.int32:
        raise ValueError("positions, slots, tables and counts must be int32")
    if len(table) != 2 or seq_blocks.shape != (table[0],):
        raise ValueError("block_table must be [S, max_blocks] and seq_blocks [S]")
    dev = q.get_device()
    for t in (k_cache, v_cache, slot_pos, block_table, seq_blocks, a, b):
        if t.get_device() != dev:
            raise ValueError("tensors must be on one device")
    if dev < 0:
        raise ValueError("tensors must be on the GPU")
    if out is None:
        out = torch.empty_like(q)
    elif out.shape != shape or out.dtype != torch.bfloat16:
        raise ValueError("O must have q's shape and type")
    elif out.get_device() != dev:
        raise ValueError("tensors must be on one device")
    if lse is None:
        lse = q.new_empty((n, Hq), dtype=torch.float32)
    elif lse.shape != (n, Hq) or lse.dtype != torch.float32:
        raise ValueError("LSE must be float32 [n, Hq]")
    elif lse.get_device() != dev:
        raise ValueError("tensors must be on one device")
    scale = 1.0 / math.sqrt(D) if softmax_scale is None else float(softmax_scale)
    return n, Hq, D, nb, Hkv, bs, table[0], table[1], out, lse, scale


def kvs_paged_decode_shared(q, k_cache, v_cache, slot_pos, block_table, seq_blocks, prefix_group, prefix_blocks,
                            softmax_scale=None, out=None, lse=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``kvs_paged_decode_shared``: ``kvs_paged_decode`` of sequences whose tables begin alike; returns (O, LSE).

    ``prefix_group`` int32 [S]: the group of each sequence (-1: none); ``prefix_blocks`` int32 [groups]: the leading
    table entries its members have in common, which are read once for all of them.
    """
    n, Hq, D, nb, Hkv, bs, S, mb, o, lse, scale = _rows_args(q, k_cache, v_cache, slot_pos, block_table, seq_blocks,
                                                             softmax_scale, out, lse, prefix_group, prefix_blocks)
    if n != S or prefix_group.shape != (S,):
        raise ValueError("q, block_table and prefix_group must have one row a sequence")
    groups = prefix_blocks.numel()
    if groups < 1 or prefix_blocks.dim() != 1:
        raise ValueError("prefix_blocks must be [groups], one group at least")
    need = lib.kvs_paged_decode_shared_workspace(S, groups, Hq, Hkv, D, mb, bs)
    ws = _workspace(need, q.device)
    with _on(q):
        _check("kvs_paged_decode_shared", lib.kvs_paged_decode_shared(
            _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(slot_pos), _ptr(block_table), _ptr(seq_blocks), _ptr(prefix_group),
            _ptr(prefix_blocks), _ptr(o), _ptr(lse), S, groups, Hq, Hkv, D, nb, bs, mb, scale, _ptr(ws), need, _stream(q)))
    return o, lse


def kvs_paged_extend(q, k_cache, v_cache, slot_pos, block_table, seq_blocks, q_pos, cu_seqlens, softmax_scale=None,
                     window: Optional[int] = None, sinks: int = 0, out=None,
                     lse=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``kvs_paged_extend``: new tokens q [Ntot, Hq, D] of S sequences over the cache that holds them; returns (O, LSE).

    Sequence s has the tokens ``cu_seqlens[s]`` to ``cu_seqlens[s + 1]`` (int32 [S + 1]), at trace positions ``q_pos``
    int32 [Ntot]; each sees the live entries at p <= its own position, under a ``window`` (None: none) those less than
    ``window`` behind it and the first ``sinks``.  LSE is float32 [Ntot, Hq].
    """
    n, Hq, D, nb, Hkv, bs, S, mb, o, lse, scale = _rows_args(q, k_cache, v_cache, slot_pos, block_table, seq_blocks,
                                                             softmax_scale, out, lse, q_pos, cu_seqlens)
    if q_pos.shape != (n,) or cu_seqlens.shape != (S + 1,):
        raise ValueError("q_pos must be [Ntot] and cu_seqlens [S + 1]")
    if window is not None and window < 1:
        raise ValueError("window must be >= 1 (None: no window)")
    need = lib.kvs_paged_extend_workspace(S, n, Hq, Hkv, D, mb, bs)
    ws = _workspace(need, q.device)
    with _on(q):
        _check("kvs_paged_extend", lib.kvs_paged_extend(
            _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(slot_pos), _ptr(block_table), _ptr(seq_blocks), _ptr(q_pos),
            _ptr(cu_seqlens), _ptr(o), _ptr(lse), S, n, Hq, Hkv, D, nb, bs, mb, scale,
            _i31(window or 0), _i31(sinks), _ptr(ws), need, _stream(q)))
    return o, lse


_SAVED_BYTES = 96 << 20   # of K and V, from which on decode() reads shared prefixes once


class PagedKVCache:
    """Device pools of a streamed paged KV cache plus its native block manager.

    ``append(seq, positions, k, v)`` stores new entries, ``evict(seq,
    positions)`` drops entries in place, ``decode(q)`` attends one query per
    sequence over the live entries of every sequence, or over those a sliding
    window shows it.  A cache made with ``weights=True`` keeps every entry's
    attention weight (``slot_weight``): entries start with the weights
    ``append`` is given, ``decode(q, accumulate=True)`` adds to them and
    ``evict_lowest(keep)`` evicts the lowest.

    ``fork(src, dst)`` lets an empty sequence share the entries of another one,
    whose common part ``decode`` reads once for all where that is faster; ``extend`` attends
    several new tokens a sequence.  ``copy(src, dst)`` gives a sequence entries
    of its own, ``compact()`` brings what evictions have left into fewer blocks.
    """

    def __init__(self, num_blocks: int, block_size: int, num_seqs: int, max_blocks: int, Hkv: int, D: int,
                 device="cuda", weights: bool = False):
        self.bm = BlockManager(num_blocks, block_size, num_seqs, max_blocks)
        self.num_blocks, self.block_size, self.num_seqs, self.max_blocks = num_blocks, block_size, num_seqs, max_blocks
        self.Hkv, self.D = Hkv, D
        self.k = torch.zeros((num_blocks, Hkv, block_size, D), dtype=torch.bfloat16, device=device)
        self.device = self.k.device   # with its index: another one may be the current one later
        self.v = torch.zeros_like(self.k)
        self.slot_pos = torch.full((num_blocks * block_size,), -1, dtype=torch.int32, device=self.device)
        self.slot_weight = torch.zeros(num_blocks * block_size, dtype=torch.float32, device=self.device) if weights else None
        self._tables = None
        self._forks = False   # whether sequences have ever shared blocks
        self._blocks = None   # of every sequence, when the tables were uploaded
        self._shares = None   # groups of sequences that share a prefix, on the device; None: not known, (): none
        self._saved = 0       # blocks the groups need not read again
        # groups of sequences by themselves; made here, as a captured decode would leave them to its graph's replays
        self._alone = (torch.full((num_seqs,), -1, dtype=torch.int32, device=self.device),
                       torch.zeros(1, dtype=torch.int32, device=self.device))

    def append(self, seq: int, positions, k_new: torch.Tensor, v_new: torch.Tensor,
               weights: Optional[torch.Tensor] = None) -> np.ndarray:
        """New entries of a sequence; ``weights`` float32 [n]: what they start with (None: 0; caches that keep weights)."""
        pos = _i32(positions)
        if k_new.shape != (pos.size, self.Hkv, self.D) or v_new.shape != k_new.shape:
            raise ValueError("k_new/v_new must be [n, Hkv, D]")
        if k_new.dtype != torch.bfloat16 or v_new.dtype != torch.bfloat16:
            raise ValueError("k_new/v_new must be bfloat16")
        if weights is not None:
            if self.slot_weight is None:
                raise ValueError("the cache keeps no weights (weights=True)")
            if weights.shape != (pos.size,) or weights.dtype != torch.float32:
                raise ValueError("weights must be float32 [n]")
            weights = weights.contiguous()
        if pos.size:   # before the manager reserves the slots
            _same_device(self.k, k_new, v_new, weights)
        slots = self.bm.append(seq, pos)
        if pos.size:
            k_new, v_new = k_new.contiguous(), v_new.contiguous()
            with _on(self.k):
                if self.slot_weight is None:
                    name = "kvs_paged_append_host"
                    st = lib.kvs_paged_append_host(_ptr(k_new), _ptr(v_new), _np_ptr(pos), _np_ptr(slots), pos.size,
                                                   _ptr(self.k), _ptr(self.v), _ptr(self.slot_pos), self.num_blocks,
                                                   self.block_size, self.Hkv, self.D, _stream(self.k))
                else:
                    name = "kvs_paged_append_weighted_host"
                    st = lib.kvs_paged_append_weighted_host(
                        _ptr(k_new), _ptr(v_new), _ptr(weights), _np_ptr(pos), _np_ptr(slots), pos.size, _ptr(self.k),
                        _ptr(self.v), _ptr(self.slot_pos), _ptr(self.slot_weight), self.num_blocks, self.block_size,
                        self.Hkv, self.D, _stream(self.k))
                if st == KVS_ERR_UNSUPPORTED:   # too many runs of slots for the launch's arguments, or under capture
                    dev_pos, dev_slots = torch.from_numpy(pos).to(self.device), torch.from_numpy(slots).to(self.device)
                    if self.slot_weight is None:
                        kvs_paged_append(k_new, v_new, dev_pos, dev_slots, self.k, self.v, self.slot_pos, self.block_size)
                    else:
                        kvs_paged_append_weighted(k_new, v_new, weights, dev_pos, dev_slots, self.k, self.v, self.slot_pos,
                                                  self.slot_weight, self.block_size)
                else:
                    _check(name, st)
        self._tables = None
        return slots

    def _mark_evicted(self, slots: np.ndarray) -> None:
        with _on(self.slot_pos):
            st = lib.kvs_paged_evict_host(_np_ptr(slots), slots.size, _ptr(self.slot_pos), self.num_blocks,
                                          self.block_size, _stream(self.slot_pos))
            if st == KVS_ERR_UNSUPPORTED:
                kvs_paged_evict(torch.from_numpy(slots).to(self.device), self.slot_pos, self.num_blocks, self.block_size)
            else:
                _check("kvs_paged_evict_host", st)

    def evict(self, seq: int, positions) -> np.ndarray:
        """Entries of a sequence leave; returns their slots, -1 for those in blocks that other sequences hold too."""
        if not (self._forks and self.bm.shared(seq) > 0):
            slots = self.bm.evict(seq, _i32(positions))
            if slots.size:
                self._mark_evicted(slots)
        else:   # what stays of a shared block goes to one of the sequence's own
            room = self._room(self.bm.live(seq))
            slots, pairs = self.bm.evict_shared(seq, positions)
            mine = slots[slots >= 0]
            if mine.size:
                self._mark_evicted(mine)
            self._copy(pairs, room)
            self._shares = None
        self._tables = None
        return slots

    def release(self, seq: int) -> np.ndarray:
        if self._forks and self.bm.shared(seq) > 0:
            self._shares = None
        slots = self.bm.release(seq)
        if slots.size:
            self._mark_evicted(slots)
        self._tables = None
        return slots

    def _room(self, entries: int) -> torch.Tensor:
        """Device memory for slots to copy from and to, asked for before the manager gives entries new slots: without it
        nothing has changed."""
        if self.k.is_cuda:
            with _on(self.k):
                if torch.cuda.is_current_stream_capturing():
                    raise RuntimeError("slots are copied by lists of the host, which a capture does not take")
        return torch.empty(2 * max(entries, 1), dtype=torch.int32, device=self.device)

    def _copy(self, pairs: np.ndarray, room: torch.Tensor, move: bool = False) -> None:
        n = pairs.shape[1]
        if n:
            room[:2 * n].copy_(torch.from_numpy(pairs.reshape(-1)))
            kvs_paged_copy(room[:n], room[n:2 * n], self.k, self.v, self.slot_pos, self.slot_weight, move)

    def fork(self, src: int, dst: int) -> None:
        """The empty sequence ``dst`` shares the entries of ``src``; what either appends or evicts then is its own."""
        if self.slot_weight is not None:
            raise ValueError("entries' weights are one sequence's: a cache that keeps them takes copy()")
        self.bm.fork(src, dst)
        self._forks = True
        self._tables = self._shares = None

    def copy(self, src: int, dst: int) -> None:
        """The empty sequence ``dst`` gets copies of the entries of ``src``, with their weights, in fresh blocks."""
        room = self._room(self.bm.live(src))
        self._copy(self.bm.copy(src, dst), room)
        self._tables = None

    def compact(self, seq: Optional[int] = None) -> int:
        """Entries of a sequence (None: of every one) move into as few blocks as hold them; returns the blocks freed.

        Blocks it shares, and a last one with room for appends, stay as they are.
        """
        before, todo, seqs = self.bm.free_blocks(), [], range(self.num_seqs) if seq is None else [seq]
        room = self._room(sum(self.bm.live(s) for s in seqs))
        try:
            for s in seqs:
                todo.append(self.bm.compact(s))
        finally:   # where the manager fails at a sequence, the entries of those in front of it have their new slots
            self._tables = None
            if todo:
                self._copy(np.concatenate(todo, axis=1), room, move=True)
        return self.bm.free_blocks() - before

    def device_tables(self) -> Tuple[torch.Tensor, torch.Tensor]:
        if self._tables is None:
            # both tables in one upload: the block counts behind the block lists
            n = self.num_seqs * self.max_blocks
            both = np.empty(n + self.num_seqs, dtype=np.int32)
            p = _np_ptr(both)
            _check("kvs_bm_tables", lib.kvs_bm_tables(self.bm._h, p, p + 4 * n))
            dev = torch.from_numpy(both).to(self.device)
            self._tables = (dev[:n].view(self.num_seqs, self.max_blocks), dev[n:])
            self._blocks = both[n:]
        return self._tables

    def device_groups(self) -> Tuple[torch.Tensor, ...]:
        """(group of every sequence, leading blocks each group has in common); empty if no sequences share their first."""
        if self._shares is None:
            group, blocks = self.bm.groups()
            self._shares, self._saved = (), 0
            if blocks.size:
                members = np.bincount(group[group >= 0], minlength=blocks.size)
                self._saved = int(((members - 1) * blocks.astype(np.int64)).sum())
                both = torch.from_numpy(np.concatenate([group, blocks])).to(self.device)
                self._shares = both[: group.size], both[group.size:]
        return self._shares

    def _pays(self) -> bool:
        saved = self._saved * 4 * self.block_size * self.Hkv * self.D
        return saved >= _SAVED_BYTES and 2 * self._saved >= int(self._blocks.sum())

    def extend(self, q: torch.Tensor, positions, lengths, softmax_scale=None, out=None, lse=None,
               window: Optional[int] = None, sinks: int = 0):
        """New tokens q [Ntot, Hq, D], ``lengths[s]`` of sequence s, at trace ``positions`` (a list, or an int32 tensor on
        the GPU), whose entries the cache holds; each sees the live entries up to its own, under a ``window`` those less
        than ``window`` behind it and the first ``sinks``.  Returns (O, LSE [Ntot, Hq])."""
        lengths = np.asarray(lengths, dtype=np.int64)
        if lengths.shape != (self.num_seqs,) or (lengths < 0).any() or lengths.sum() != q.shape[0]:
            raise ValueError("lengths must be one number a sequence, q's rows in all")
        table, nblk = self.device_tables()
        cu = torch.from_numpy(_i32(np.concatenate([[0], np.cumsum(lengths)]))).to(self.device)
        if not torch.is_tensor(positions):
            positions = torch.from_numpy(_i32(positions)).to(self.device)
        return kvs_paged_extend(q, self.k, self.v, self.slot_pos, table, nblk, positions, cu, softmax_scale, window, sinks,
                                out, lse)

    def decode(self, q: torch.Tensor, softmax_scale=None, out=None, lse=None, positions=None,
               window: Optional[int] = None, sinks: int = 0, accumulate: bool = False):
        """One query a sequence, q [num_seqs, Hq, D]; returns (O, LSE).

        ``window`` (with ``positions``, the queries' trace positions: a list or an int32 tensor on the GPU) shows each
        query the entries less than ``window`` behind it and the first ``sinks``; without a window every live entry is
        seen, and ``positions`` and ``sinks`` have no effect (layers of both kinds take the same call).  ``accumulate``
        adds the entries' attention weights to ``slot_weight``.  A KV head may have 64 q-heads, with a window or
        ``accumulate`` 32.  Where a prefix that more than 128 of a KV head's rows share (D = 64: 64; sequences times q-heads)
        is read once, O is 2.3e-3 off the exact result in the 2-norm, elsewhere 2.0e-3.
        """
        table, nblk = self.device_tables()
        if window is None and not accumulate:
            shares = self.device_groups() if self._forks else ()
            # Reading a shared prefix once takes two or three launches more than reading it once a sequence, mostly from the
            # caches.  32/8 heads, D = 128: 16 sequences behind 4,096 entries with 1,000 of their own 49 -> 36 us, 8 behind
            # 4,096 with 500 26 -> 25; but 64 behind 1,024 with 1,000 67 -> 73, 8 behind 2,048 with 500 19 -> 23.  The line is
            # drawn by these; it does not know what planning many sequences takes (1,024 in 128 groups 381 -> 459).
            # More than 32 q-heads a KV head the plain call does not take, whatever is shared.
            many = q.dim() == 3 and q.shape[1] > 32 * self.Hkv
            if many or (shares and self._pays()):
                return kvs_paged_decode_shared(q, self.k, self.v, self.slot_pos, table, nblk, *(shares or self._alone),
                                               softmax_scale, out, lse)
            with _on(self.k):
                return kvs_paged_decode(q, self.k, self.v, self.slot_pos, table, nblk, softmax_scale, out, lse)
        if accumulate and self.slot_weight is None:
            raise ValueError("the cache keeps no weights (weights=True)")
        if positions is not None and not torch.is_tensor(positions):
            positions = torch.from_numpy(_i32(positions)).to(self.device)
        return kvs_paged_decode_ex(q, self.k, self.v, self.slot_pos, table, nblk, softmax_scale, positions, window,
                                   sinks, self.slot_weight if accumulate else None, out, lse)

    def evict_lowest(self, keep, sinks: int = 0, recent: int = 0):
        """Evict the entries of lowest weight of every sequence that holds more than ``keep`` (one number, or one a
        sequence); positions below ``sinks`` and the ``recent`` newest stay.  Returns the evicted positions of every
        sequence (waits for the GPU, which picks them)."""
        if self.slot_weight is None:
            raise ValueError("the cache keeps no weights (weights=True)")
        if sinks < 0 or recent < 0:
            raise ValueError("sinks and recent must be >= 0")
        want = np.broadcast_to(np.maximum(np.asarray(keep, dtype=np.int64), 0), (self.num_seqs,))
        over = max(self.bm.live(s) - int(want[s]) for s in range(self.num_seqs))
        if over <= 0:
            return [np.empty(0, dtype=np.int32) for _ in range(self.num_seqs)]
        table, nblk = self.device_tables()
        dev_keep = torch.from_numpy(np.minimum(want, 0x7FFFFFFF).astype(np.int32)).to(self.device)
        pos, counts = kvs_paged_evict_lowest(self.slot_weight, self.slot_pos, table, nblk, dev_keep, self.block_size,
                                             sinks, recent, over)
        n, rows = counts.cpu().numpy(), pos.cpu().numpy()
        gone = [rows[s, : n[s]].copy() for s in range(self.num_seqs)]
        for s, p in enumerate(gone):
            if p.size:
                self.bm.evict(s, p)
        self._tables = None
        return gone
