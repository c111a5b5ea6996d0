"""Which form PagedKVCache.decode takes (MI355X): results are the same whether a shared prefix is read once or once a
sequence, on the groups that the cache keeps itself, and heads of more than 32 to a KV head decode in every state."""
import math

import pytest
import torch

from tests import test_gpu_paged_share as share
from tests.gpu_helpers import announce

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pg():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import paged

    return paged


@pytest.fixture(params=["any saving pays", "sharing is always taken"])
def taken(pg, request, monkeypatch):
    """The calls of decode() that read a prefix once, under a lower threshold or none."""
    calls, pays = [], pg.PagedKVCache._pays
    if request.param == "any saving pays":
        monkeypatch.setattr(pg, "_SAVED_BYTES", 0)
        monkeypatch.setattr(pg.PagedKVCache, "_pays", lambda c: calls.append(pays(c)) or calls[-1])
    else:
        monkeypatch.setattr(pg.PagedKVCache, "_pays", lambda c: calls.append(True) or True)
    return calls


@pytest.mark.parametrize("case", [share.DECODE[i] for i in (2, 3, 4, 6, 8, 10)], ids=lambda c: f"{len(c[0])}_H{c[2]}x{c[3]}_D{c[4]}")
def test_decode_over_shared_prefixes(pg, taken, case):
    share.test_decode_over_shared_prefixes(pg, case)
    assert taken or case[2] > 32 * case[3]       # which do not ask


@pytest.mark.parametrize("block", [1, 5, 16])
def test_life_of_two_groups(pg, taken, block):
    share.test_life_of_two_groups(pg, block)
    assert taken[0]       # block size 1: 514 of the 718 blocks held are read again otherwise; 104 of 151, 34 of 54


@pytest.mark.parametrize("D", [64, 128])
def test_many_heads_of_a_kv_head_in_every_state(pg, D):
    """64 q-heads a KV head: before a fork, while blocks are shared, behind the last shared one, and in a cache that keeps
    weights, which cannot fork."""
    announce(f"decode of 64 q-heads a KV head, D {D}")
    scale = 1 / math.sqrt(D)
    for weights in (False, True):
        r = share.Rollouts(pg, 3, 60, 16, 30, 1, D, 5, weights=weights)
        q = r.randn(3, 64, D)

        def check(name):
            o, lse = r.cache.decode(q.to(share.DEV))
            r.check_decode(name, q, o, lse, scale)

        check("empty")
        r.append(0, range(100))
        check("before a fork")
        if not weights:
            r.fork(0, 1)
            r.append(1, range(100, 140))
            check("shared")
            r.evict(1, range(100))
            check("evicted apart")
            r.fork(0, 2)
            r.cache.release(0)
            r.held[0] = {}
            check("released")
        with pytest.raises(pg.KvsError):         # a window and weights take 32
            r.cache.decode(q.to(share.DEV), positions=[140] * 3, window=50)
