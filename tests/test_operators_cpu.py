"""Windows, weights and evictions without a GPU: the plain forms agree with brute force, the calls refuse bad arguments
before any HIP call, workspace sizes follow the documentation, and the bindings refuse mismatched tensors."""
import os

import numpy as np
import pytest
import torch

from tests import operators_ref as ref

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_35750_amd", "libkvs.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libkvs.so not built (run __graft_entry__.build())")
FAKE = 1 << 20   # 16-byte aligned, never dereferenced: validation fails first
OK, NULL, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 7


@pytest.fixture(scope="module")
def kvs():
    from paper_2609_35750_amd import kvs as k

    return k


@pytest.fixture(scope="module")
def paged():
    from paper_2609_35750_amd import paged as p

    return p


# ---------------------------------------------------------------- the plain forms
@pytest.mark.parametrize("L,window,sinks", [(1, 1, 0), (7, 1, 0), (9, 3, 2), (20, 5, 30), (33, 64, 0), (40, 8, 11)])
@pytest.mark.parametrize("evict", [False, True])
def test_window_is_an_eviction_index(L, window, sinks, evict):
    """min(e_j, j + W) for j >= S reproduces the window's mask, row by row."""
    e = np.random.default_rng(L).integers(np.arange(L) + 1, L + 3) if evict else None
    see = ref.mask(L, window, sinks, e)
    u = ref.until(L, window, sinks, e)
    i, j = np.arange(L)[:, None], np.arange(L)[None, :]
    np.testing.assert_array_equal(see, (j <= i) & (i < u[None, :]))
    full = np.minimum(np.arange(L) + window, L)
    full = np.where(np.arange(L) < sinks, L, full)
    np.testing.assert_array_equal(u, full if e is None else np.minimum(full, e))
    assert see.diagonal().all()


def test_weights_of_a_trace_sum_to_its_rows():
    """Every row of the softmax sums to 1, so all weights sum to rows x heads."""
    rng = np.random.default_rng(0)
    q, k = rng.normal(size=(30, 4, 8)), rng.normal(size=(30, 2, 8))
    see = ref.mask(30, 7, 2)
    lse = np.stack([np.log(np.where(see, np.exp(0.3 * q[:, h] @ k[:, h // 2].T), 0).sum(1)) for h in range(4)])
    w, _ = ref.key_weights(q, k, lse, 0.3, 7, 2)
    assert abs(w.sum() - 120.0) < 1e-9
    w, _ = ref.key_weights(q, k, lse, 0.3, 7, 2, last_rows=5)
    assert abs(w.sum() - 20.0) < 1e-9


def test_evict_lowest_by_hand():
    pos = np.array([0, 1, -1, 3, 4, 5, 6, 7], dtype=np.int32)
    w = np.array([0.0, 5.0, 0.0, 1.0, 1.0, np.nan, -0.0, 0.0])
    args = (np.array([1, 0]), 2, 4, 2)      # blocks 1, 0 of four slots: table order 4 5 6 7 0 1 3
    assert ref.evict_lowest(w, pos, *args, keep=5, sinks=1, recent=1, max_out=9) == [4, 6]
    assert ref.evict_lowest(w, pos, *args, keep=0, sinks=0, recent=0, max_out=3) == [6, 7, 0]
    assert ref.evict_lowest(w, pos, *args, keep=0, sinks=0, recent=2, max_out=9) == [4, 5, 0, 1, 3]
    assert ref.evict_lowest(w, pos, *args, keep=7, sinks=0, recent=0, max_out=9) == []


# ---------------------------------------------------------------- C refusals
def _wfwd(kvs, cu=None, B=2, N=120, T=60, Hq=4, Hkv=2, D=64, scale=0.1, window=8, sinks=2, q=FAKE, o=FAKE, ws=FAKE,
          ws_bytes=None):
    need = kvs.lib.kvs_window_attn_fwd_workspace(B, N, T, Hq, Hkv, D) if ws_bytes is None else ws_bytes
    return kvs.lib.kvs_window_attn_fwd(q, FAKE, FAKE, None, cu, o, FAKE, B, N, T, Hq, Hkv, D, scale, window, sinks, ws,
                                       need, None)


def test_window_forward_refusals(kvs):
    assert _wfwd(kvs, window=0) == SHAPE and b"window" in kvs.lib.kvs_last_error()
    assert _wfwd(kvs, window=-3) == SHAPE
    assert _wfwd(kvs, sinks=-1) == SHAPE
    assert _wfwd(kvs, N=100) == SHAPE                  # 2 x 60 tokens without cu_seqlens
    assert _wfwd(kvs, D=96) == SHAPE and _wfwd(kvs, Hq=5) == SHAPE and _wfwd(kvs, scale=float("nan")) == SHAPE
    assert _wfwd(kvs, B=1, N=(1 << 20) + 1, T=(1 << 20) + 1) == UNSUPPORTED
    assert _wfwd(kvs, q=None) == NULL and _wfwd(kvs, o=FAKE + 4) == ALIGN
    assert _wfwd(kvs, ws_bytes=8) == WORKSPACE and _wfwd(kvs, ws=None) == NULL and _wfwd(kvs, ws=FAKE + 16) == ALIGN
    # an empty batch looks at no pointer
    assert kvs.lib.kvs_window_attn_fwd(None, None, None, None, FAKE, None, None, 3, 0, 1, 4, 2, 64, 0.1, 8, 2, None, 0,
                                       None) == OK


def test_window_backward_refusals(kvs):
    L = kvs.lib
    need = L.kvs_window_attn_bwd_workspace(2, 120, 60, 4, 2, 64)
    assert need > L.kvs_evict_attn_bwd_workspace(2, 60, 4, 2, 64)      # and the keys' last visible queries

    def bwd(window=8, sinks=2, dq=FAKE, lse=FAKE, ws_bytes=need, N=120):
        return L.kvs_window_attn_bwd(FAKE, FAKE, FAKE, FAKE, FAKE, lse, None, None, dq, FAKE, FAKE, 2, N, 60, 4, 2, 64,
                                     0.1, window, sinks, FAKE, ws_bytes, None)
    assert bwd(window=0) == SHAPE and bwd(sinks=-1) == SHAPE and bwd(N=119) == SHAPE
    assert bwd(dq=None) == NULL and bwd(lse=FAKE + 8) == ALIGN
    assert bwd(ws_bytes=120 * 4) == WORKSPACE


def test_key_weights_refusals(kvs):
    L = kvs.lib

    def kw(window=0, sinks=0, rows=0, w=FAKE, B=2, N=120, T=60, ws_bytes=None, lse=FAKE):
        need = L.kvs_key_weights_workspace(B, N, T, 4, 2, 64, rows) if ws_bytes is None else ws_bytes
        return L.kvs_key_weights(FAKE, FAKE, lse, None, None, w, B, N, T, 4, 2, 64, 0.1, window, sinks, rows, FAKE, need,
                                 None)
    assert kw(window=-1) == SHAPE and kw(sinks=-1) == SHAPE and kw(rows=-1) == SHAPE and kw(N=7) == SHAPE
    assert kw(w=None) == NULL and kw(lse=FAKE + 4) == ALIGN and kw(ws_bytes=64) == WORKSPACE
    assert L.kvs_key_weights(None, None, None, None, FAKE, None, 3, 0, 1, 4, 2, 64, 0.1, 0, 0, 0, None, 0, None) == OK
    # fewer rows never take more room
    sizes = [L.kvs_key_weights_workspace(1, 16384, 16384, 32, 8, 128, r) for r in (1, 64, 4096, 16384, 0)]
    assert sizes[-1] == sizes[-2] and all(s > 0 for s in sizes)


def test_decode_ex_refusals(kvs):
    L = kvs.lib

    def dec(window=8, sinks=2, q_pos=FAKE, weight=FAKE, S=3, Hq=4, Hkv=2, D=64, nb=9, bs=16, mb=5, ws=FAKE, short=0,
            table=FAKE):
        need = L.kvs_paged_decode_ex_workspace(S, Hq, Hkv, D, nb, mb, bs, window, sinks, weight is not None)
        return L.kvs_paged_decode_ex(FAKE, FAKE, FAKE, FAKE, weight, table, FAKE, q_pos, FAKE, FAKE, S, Hq, Hkv, D, nb,
                                     bs, mb, 0.1, window, sinks, ws, need - short, None)
    assert dec(window=-1) == SHAPE and dec(sinks=-1) == SHAPE and dec(bs=65) == SHAPE and dec(D=32) == SHAPE
    assert dec(q_pos=None) == NULL and b"q_pos" in L.kvs_last_error()
    assert dec(table=None) == NULL
    assert dec(short=1) == WORKSPACE and dec(ws=None) == NULL
    assert dec(Hq=66, Hkv=2) == UNSUPPORTED
    assert dec(S=65536, weight=None) == UNSUPPORTED
    assert dec(mb=1 << 27, weight=None) == UNSUPPORTED
    # a window bounds what a call needs, whatever the table's width
    wide = L.kvs_paged_decode_ex_workspace(64, 32, 8, 128, 10000, 1 << 16, 16, 1024, 4, 1)
    assert wide < 256 << 20
    assert L.kvs_paged_decode_ex_workspace(0, 4, 2, 64, 9, 5, 16, 0, 0, 0) == 0


def test_evict_lowest_refusals(kvs):
    L = kvs.lib

    def ev(S=3, nb=9, bs=16, mb=5, sinks=0, recent=0, most=4, keep=FAKE, ws=None, ws_bytes=0):
        return L.kvs_paged_evict_lowest(FAKE, FAKE, FAKE, FAKE, keep, FAKE, FAKE, S, nb, bs, mb, sinks, recent, most, ws,
                                        ws_bytes, None)
    assert ev(S=0) == SHAPE and ev(bs=0) == SHAPE and ev(most=0) == SHAPE and ev(sinks=-1) == SHAPE and ev(recent=-1) == SHAPE
    assert ev(keep=None) == NULL
    assert ev(mb=1 << 27) == UNSUPPORTED and ev(S=65536) == UNSUPPORTED and ev(S=60000, mb=1 << 16, bs=64) == UNSUPPORTED
    assert L.kvs_paged_evict_lowest_workspace(3, 5, 16) == 0
    need = L.kvs_paged_evict_lowest_workspace(3, 5000, 1)
    assert need >= 3 * 5000 * 8
    assert ev(bs=1, mb=5000) == NULL and ev(bs=1, mb=5000, ws=FAKE, ws_bytes=need - 1) == WORKSPACE


def test_append_weighted_refusals(kvs):
    L = kvs.lib

    def ap(fn, weight=FAKE, n=2, k=FAKE, D=64):
        return fn(k, FAKE, None, FAKE, FAKE, n, FAKE, FAKE, FAKE, weight, 4, 16, 2, D, None)
    for fn in (L.kvs_paged_append_weighted, L.kvs_paged_append_weighted_host):
        assert ap(fn, weight=None) == NULL and ap(fn, k=None) == NULL and ap(fn, D=65) == SHAPE and ap(fn, n=-1) == SHAPE
        assert ap(fn, n=0) == OK


# ---------------------------------------------------------------- the bindings' refusals
def test_binding_refuses_mismatches(kvs, paged):
    b16 = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    q, k = b16(1, 8, 4, 64), b16(1, 8, 2, 64)
    lse = torch.zeros(1, 4, 8)
    for bad in (dict(q=q.float()), dict(v=b16(1, 8, 2, 32)), dict(k=b16(1, 7, 2, 64), v=b16(1, 7, 2, 64)),
                dict(evict_at=torch.zeros(1, 8)), dict(evict_at=torch.zeros(8, dtype=torch.int32)), {}):
        a = dict(dict(q=q, k=k, v=k), **bad)      # the last one: tensors on the CPU
        with pytest.raises(ValueError):
            kvs.kvs_window_attn_fwd(a["q"], a["k"], a["v"], 4, 0, a.get("evict_at"))
    with pytest.raises(ValueError, match="max_seqlen"):
        kvs.kvs_window_attn_fwd(b16(8, 4, 64), b16(8, 2, 64), b16(8, 2, 64), 4, 0,
                                cu_seqlens=torch.tensor([0, 8], dtype=torch.int32))
    with pytest.raises(ValueError, match="window"):
        kvs.kvs_key_weights(q, k, lse, window=0)
    with pytest.raises(ValueError, match="last_rows"):
        kvs.kvs_key_weights(q, k, lse, last_rows=0)
    with pytest.raises(ValueError):
        kvs.kvs_key_weights(q, k, lse.double())
    kc, pos = b16(3, 2, 16, 64), torch.zeros(48, dtype=torch.int32)
    table, nblk = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    q1 = b16(1, 4, 64)
    for kw in (dict(window=0, q_pos=nblk), dict(window=4), dict(window=4, q_pos=nblk.long()),
               dict(window=4, q_pos=torch.zeros(2, dtype=torch.int32)), dict(slot_weight=torch.zeros(47)),
               dict(slot_weight=torch.zeros(48).double()), dict(out=b16(1, 4, 32)), dict(lse=torch.zeros(1, 3)), {}):
        with pytest.raises(ValueError):
            paged.kvs_paged_decode_ex(q1, kc, kc, pos, table, nblk, **kw)
    for a in ((torch.zeros(47), pos, table, nblk, nblk, 16), (torch.zeros(48), pos, table, nblk, nblk.long(), 16),
              (torch.zeros(48), pos, table, nblk, nblk, 5), (torch.zeros(48), pos, table, nblk, nblk, 16)):
        with pytest.raises(ValueError):
            paged.kvs_paged_evict_lowest(*a)


def test_cache_without_weights_refuses(paged):
    cache = paged.PagedKVCache(4, 16, 1, 2, 2, 64, device="cpu")
    with pytest.raises(ValueError, match="weights"):
        cache.decode(torch.zeros(1, 4, 64, dtype=torch.bfloat16), accumulate=True)
    with pytest.raises(ValueError, match="weights"):
        cache.evict_lowest(3)
    with pytest.raises(ValueError, match="weights"):
        cache.append(0, [0], torch.zeros(1, 2, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 64, dtype=torch.bfloat16),
                     weights=torch.zeros(1))
    assert cache.bm.live(0) == 0
    cache = paged.PagedKVCache(4, 16, 2, 2, 2, 64, device="cpu", weights=True)
    assert [g.size for g in cache.evict_lowest(0)] == [0, 0]      # nothing is cached: nothing to do
    with pytest.raises(ValueError):
        cache.evict_lowest(0, sinks=-1)


# ---------------------------------------------------------------- captured backward
def test_backward_under_capture_refuses_leaves_of_an_eager_graph(kvs):
    """The leaf's node is marked while a graph made on the default stream lives, through other nodes it is not looked
    for, and the mark goes with the graph."""
    x, w = torch.ones(3, requires_grad=True), torch.ones(3, requires_grad=True)
    eager = x * w
    kvs._mark_eager(eager)
    with pytest.raises(RuntimeError, match="captured"):
        kvs._refuse_captured((x * 2.0).grad_fn.next_functions)
    kvs._refuse_captured(((x * 2.0) * 3.0).grad_fn.next_functions)
    kvs._refuse_captured(torch.ones(2, requires_grad=True).exp().grad_fn.next_functions)
    del eager
    kvs._refuse_captured((x * 2.0).grad_fn.next_functions)


def test_scales_that_are_not_finite(kvs):
    for scale in (float("inf"), float("-inf"), float("nan"), 0.0, -1.0):
        assert _wfwd(kvs, scale=scale) == SHAPE, scale


def test_remainders_are_checked(kvs):
    L, need = kvs.lib, kvs.lib.kvs_window_attn_bwd_workspace(2, 120, 60, 4, 2, 64)
    assert L.kvs_window_attn_fwd_rem(FAKE, FAKE, FAKE, None, None, FAKE, FAKE + 8, FAKE, 2, 120, 60, 4, 2, 64, 0.1, 8, 2,
                                     FAKE, need, None) == ALIGN
    assert L.kvs_window_attn_bwd_rem(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE + 4, FAKE, None, None, FAKE, FAKE, FAKE, 2, 120, 60,
                                     4, 2, 64, 0.1, 8, 2, FAKE, need, None) == ALIGN
    q = torch.zeros(1, 8, 4, 64).bfloat16()
    with pytest.raises(ValueError, match="int8"):
        kvs._rem_like(torch.zeros(1, 8, 4, 64), q)
    with pytest.raises(ValueError, match="shape"):
        kvs._rem_like(torch.zeros(1, 8, 2, 64, dtype=torch.int8), q)
