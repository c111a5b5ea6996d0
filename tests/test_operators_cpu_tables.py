"""Workspaces of the weighted decode under tables that list entries outside the cache (no GPU)."""
import os

import pytest

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_35750_amd", "libkvs.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libkvs.so not built (run __graft_entry__.build())")


@pytest.fixture(scope="module")
def lib():
    from paper_2609_35750_amd import kvs

    return kvs.lib


def _scores(lib, S, Hq, Hkv, D, nb, mb, bs, window):
    """Bytes the weights add to a call's workspace."""
    return (lib.kvs_paged_decode_ex_workspace(S, Hq, Hkv, D, nb, mb, bs, window, 0, 1) -
            lib.kvs_paged_decode_ex_workspace(S, Hq, Hkv, D, nb, mb, bs, window, 0, 0))


@pytest.mark.parametrize("S,mb", [(1, 12), (4, 60), (20, 8)])
def test_picked_slots_have_rows_for_all_listed_tiles(lib, S, mb):
    """Four blocks of 16 slots, tables of many more entries: every tile a wave may pick from has its scores and slots."""
    tiles = S * -(-mb * 16 // 32)
    assert tiles > 4 * 16 // 32 + S
    assert _scores(lib, S, 4, 2, 128, 4, mb, 16, 8) >= tiles * 32 * 4 * (4 + 1)


def test_without_a_window_one_row_more_than_the_cache_fills(lib):
    """A row takes the scores of all tiles beyond those the cache's slots make; wide tables cost nothing more."""
    row = 4 * 32 * 4
    rows = 4 * 16 // 32 + 1
    assert (rows + 1) * row <= _scores(lib, 1, 4, 2, 128, 4, 12, 16, 0) < (rows + 2) * row + 256
    assert _scores(lib, 1, 4, 2, 128, 4, 12, 16, 0) == _scores(lib, 1, 4, 2, 128, 4, 1 << 16, 16, 0)


def test_more_tiles_than_31_bits_number_are_refused(lib):
    """Tables as wide as 65,536 sequences of 2^20 slots: their tiles' numbers would leave 32-bit integers."""
    fake = 1 << 20

    def dec(S, mb, weight, window=0):
        need = lib.kvs_paged_decode_ex_workspace(S, 4, 1, 64, 64, mb, 64, window, 0, weight is not None)
        return lib.kvs_paged_decode_ex(fake, fake, fake, fake, weight, fake, fake, fake if window else None, None, fake, S, 4,
                                       1, 64, 64, 64, mb, 0.1, window, 0, fake, need, None)
    null, unsupported = 1, 7      # with everything else in order the missing O is what is found
    assert dec(65536, 1 << 14, fake) == unsupported and b"tiles" in lib.kvs_last_error()
    assert dec(65535, 1 << 14, fake) == null
    assert dec(65536, 1 << 14, None) == null            # without weights no tile is numbered
    assert dec(64, 1 << 24, fake, 1 << 30) == unsupported
    assert dec(64, 1 << 24, fake, 4096) == null         # the window bounds what is listed


def test_counts_beyond_32_bits_are_refused_not_cut():
    """A list of 2^32 + 5 positions would be taken for one of 5, its rows for rows of 5."""
    import torch

    from paper_2609_35750_amd import paged

    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    for most in (1 << 31, (1 << 32) + 5):
        with pytest.raises(ValueError, match="max_out"):
            paged.kvs_paged_evict_lowest(torch.zeros(48), i32(48), i32(1, 2), i32(1), i32(1), 16, max_out=most)


def test_weighted_append_checks_the_caches():
    """Entries of other sizes or types than the cache's would be read and written out of range."""
    import torch

    from paper_2609_35750_amd import paged

    b16 = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    good = dict(k_new=b16(3, 2, 64), v_new=b16(3, 2, 64), k_cache=b16(4, 2, 16, 64), v_cache=b16(4, 2, 16, 64),
                slot_pos=i32(64), block_size=16)
    for bad, match in ((dict(k_new=b16(3, 4, 64), v_new=b16(3, 4, 64)), "Hkv"), (dict(v_cache=b16(4, 1, 16, 64)), "Hkv"),
                       (dict(k_new=b16(3, 2, 128), v_new=b16(3, 2, 128)), "Hkv"), (dict(slot_pos=i32(63)), "slot_pos"),
                       (dict(k_new=torch.zeros(3, 2, 64, dtype=torch.int8)), "bfloat16"),
                       (dict(v_cache=torch.zeros(4, 2, 16, 64)), "bfloat16"), ({}, "GPU")):
        a = {**good, **bad}
        with pytest.raises(ValueError, match=match):
            paged.kvs_paged_append_weighted(a["k_new"], a["v_new"], None, i32(3), i32(3), a["k_cache"], a["v_cache"],
                                            a["slot_pos"], torch.zeros(64), a["block_size"])
    for weights in (False, True):
        cache = paged.PagedKVCache(4, 16, 1, 2, 2, 64, device="cpu", weights=weights)
        with pytest.raises(ValueError, match="bfloat16"):
            cache.append(0, [0, 1, 2], b16(3, 2, 64), torch.zeros(3, 2, 64, dtype=torch.int8))
        assert cache.bm.live(0) == 0


def test_refused_append_leaves_the_manager_as_it_was():
    """Tensors that are not where the cache is are refused before slots are reserved for them."""
    import torch

    from paper_2609_35750_amd import paged

    cache = paged.PagedKVCache(4, 16, 1, 2, 2, 64, device="cpu", weights=True)
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    for w in (None, torch.zeros(3)):
        with pytest.raises(ValueError, match="GPU"):
            cache.append(0, [0, 1, 2], k, k, weights=w)
        assert cache.bm.live(0) == 0 and cache.bm.free_blocks() == 4
    cache.k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16, device="meta")
    with pytest.raises(ValueError, match="one device"):
        cache.append(0, [0, 1, 2], k, k)
    assert cache.bm.live(0) == 0


def test_cache_calls_run_with_its_device_current(monkeypatch):
    """Every call of a cache into the library is made with the cache's device as the current one."""
    import contextlib

    import numpy as np
    import torch

    from paper_2609_35750_amd import paged

    inside, calls = [0], []

    @contextlib.contextmanager
    def on(t):
        inside[0] += 1
        yield
        inside[0] -= 1

    class Lib:
        """The library's host side; its calls for the GPU are recorded. Host lists are declined, so that the
        calls behind them are seen too."""
        def __getattr__(self, name):
            real = getattr(paged_lib, name)
            if name.startswith("kvs_bm_") or name.endswith("_workspace"):
                return real

            def call(*a):
                calls.append((name, inside[0]))
                return paged.KVS_ERR_UNSUPPORTED if name.endswith("_host") else 0
            return call
    paged_lib = paged.lib
    cache = paged.PagedKVCache(8, 16, 1, 8, 2, 64, device="cpu", weights=True)
    plain = paged.PagedKVCache(8, 16, 1, 8, 2, 64, device="cpu")
    for name, to in (("lib", Lib()), ("_on", on), ("_ptr", lambda t: 1 << 20), ("_stream", lambda t: 0),
                     ("_same_device", lambda *t: None)):
        monkeypatch.setattr(paged, name, to)
    k, q = torch.zeros(30, 2, 64, dtype=torch.bfloat16), torch.zeros(1, 4, 64, dtype=torch.bfloat16)
    for c in (cache, plain):
        c.append(0, np.arange(30), k, k)
        c.evict(0, [3, 5])
        c.decode(q)
        c.decode(q, positions=[30], window=8)
    cache.decode(q, accumulate=True)
    pos, counts = torch.tensor([[1, 2]], dtype=torch.int32), torch.tensor([2], dtype=torch.int32)
    made = paged.kvs_paged_evict_lowest
    monkeypatch.setattr(paged, "kvs_paged_evict_lowest", lambda *a: (made(*a), (pos, counts))[1])
    assert [g.tolist() for g in cache.evict_lowest(26)] == [[1, 2]]
    for c in (cache, plain):
        c.release(0)
    names = {n for n, _ in calls}
    assert names >= {"kvs_paged_append_host", "kvs_paged_append", "kvs_paged_append_weighted_host",
                     "kvs_paged_append_weighted", "kvs_paged_evict_host", "kvs_paged_evict", "kvs_paged_decode",
                     "kvs_paged_decode_ex", "kvs_paged_evict_lowest"}
    assert all(depth >= 1 for _, depth in calls), [n for n, depth in calls if depth < 1]


def test_lengths_beyond_32_bits_are_not_cut(monkeypatch):
    """A bound of 2^32 + 4 tokens would be taken for one of 4, and every trace cut to it."""
    import torch

    from paper_2609_35750_amd import kvs

    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    q, k = torch.zeros(8, 4, 64, dtype=torch.bfloat16), torch.zeros(8, 2, 64, dtype=torch.bfloat16)
    cu = torch.tensor([0, 8], dtype=torch.int32)
    for mx, T in ((8, 8), ((1 << 32) + 4, 2 ** 31 - 1), (1 << 31, 2 ** 31 - 1)):
        got = kvs._window_args((), (), (), q, k, None, cu, mx, None, True)
        assert got[2] == T
    # the calls refuse such a bound, and the queries do not compute with it
    assert kvs.lib.kvs_window_attn_bwd_workspace(1, 8, 2 ** 31 - 1, 4, 2, 64) == 0
    assert kvs.lib.kvs_key_weights_workspace(1, 8, 2 ** 31 - 1, 4, 2, 64, 0) == 0
    fake = 1 << 20
    assert kvs.lib.kvs_window_attn_bwd(fake, fake, fake, fake, fake, fake, None, fake, fake, fake, fake, 1, 8, 2 ** 31 - 1, 4,
                                       2, 64, 0.1, 8, 0, fake, 0, None) == 7
    assert kvs.lib.kvs_key_weights(fake, fake, fake, None, fake, fake, 1, 8, 2 ** 31 - 1, 4, 2, 64, 0.1, 0, 0, 0, fake, 0,
                                   None) == 7


def test_stream_handle_without_the_private_name(monkeypatch):
    """A torch that lacks the name for the raw handle gives the same stream through its public calls."""
    import types

    import torch

    from paper_2609_35750_amd import kvs

    t = types.SimpleNamespace(device=types.SimpleNamespace(index=3))
    monkeypatch.setattr(kvs, "_RAW_STREAM", lambda i: 100 + i)
    assert kvs._stream(t) == 103
    monkeypatch.setattr(kvs, "_RAW_STREAM", None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d: types.SimpleNamespace(cuda_stream=200 + d.index))
    assert kvs._stream(t) == 203


def test_eviction_limits_are_the_documented_ones(lib):
    """num_seqs * (max_blocks * block_size + 255) below 2^32, at the line."""
    fake = 1 << 20

    def ev(S, mb):
        return lib.kvs_paged_evict_lowest(fake, fake, fake, fake, None, fake, fake, S, 64, 1, mb, 0, 0, 4, None, 0, None)
    null, unsupported = 1, 7      # keep is missing: what is found when the sizes are in order
    for S in (1, 5, 65535):
        mb = min((2 ** 32 - 1) // S - 255, 1 << 30)
        assert ev(S, mb) == null and ev(S, mb + 1) == unsupported
