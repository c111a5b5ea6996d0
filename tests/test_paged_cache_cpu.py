"""PagedKVCache on the host: which form of the decode it takes (no GPU; the calls into the library are recorded)."""
import contextlib
import os

import pytest
import torch

LIB = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_35750_amd", "libkvs.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libkvs.so not built (run __graft_entry__.build())")


@pytest.fixture
def paged(monkeypatch):
    from paper_2609_35750_amd import paged as p

    monkeypatch.setattr(p, "_on", lambda t: contextlib.nullcontext())
    return p


@pytest.fixture
def decodes(paged, monkeypatch):
    """Form and groups of every decode."""
    calls = []
    monkeypatch.setattr(paged, "kvs_paged_decode", lambda *a: calls.append(("plain",)))
    monkeypatch.setattr(paged, "kvs_paged_decode_shared",
                        lambda *a: calls.append(("shared", a[6].tolist(), a[7].tolist())))
    return calls


def _cache(paged, weights=False):
    return paged.PagedKVCache(40, 4, 3, 20, 2, 64, device="cpu", weights=weights)


def test_many_heads_decode_in_every_state(paged, decodes):
    """64 q-heads a KV head take the call for shared prefixes before a fork, while blocks are shared and behind that."""
    many, few = (torch.zeros(3, h, 64, dtype=torch.bfloat16) for h in (128, 64))

    def forms(cache):
        decodes.clear()
        cache.decode(many)
        cache.decode(few)
        assert decodes[1] == ("plain",)      # nothing here saves enough
        return decodes[0]

    alone = ("shared", [-1, -1, -1], [0])
    cache = _cache(paged)
    assert forms(cache) == alone
    cache.bm.append(0, range(10))
    assert forms(cache) == alone
    cache.fork(0, 2)
    assert forms(cache) == ("shared", [0, -1, 0], [3])
    cache.bm.evict(2, range(10))             # its device side has no GPU here
    cache._tables = cache._shares = None
    assert forms(cache) == alone
    cache = _cache(paged, weights=True)      # which do not fork
    cache.bm.append(1, range(10))
    assert forms(cache) == alone


def test_saved_reads_decide(paged, decodes, monkeypatch):
    """The shared form from _SAVED_BYTES of K and V on, where they are half of all; groups follow what sequences hold."""
    cache = _cache(paged)
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    cache.bm.append(0, range(12))
    cache.fork(0, 1)
    cache.fork(0, 2)
    saved = 2 * 3 * 4 * 2 * 64 * 4           # two sequences, three blocks of four entries, K and V of two heads
    for least, form in ((saved, "shared"), (saved + 1, "plain")):
        monkeypatch.setattr(paged, "_SAVED_BYTES", least)
        cache.decode(q)
        assert decodes.pop()[0] == form
    monkeypatch.setattr(paged, "_SAVED_BYTES", 0)
    cache.bm.append(1, range(12, 24))        # 6 of 12 blocks need no second reading, then 6 of 13
    cache._tables = None
    cache.decode(q)
    assert decodes.pop() == ("shared", [0, 0, 0], [3])
    cache.bm.append(2, [12])
    cache._tables = None
    cache.decode(q)
    assert decodes.pop() == ("plain",)
