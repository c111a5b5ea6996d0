"""Copies of a cache's entries under a capture (MI355X): refused before anything changes, and the capture goes on."""
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


def test_copies_are_not_captured(pg):
    announce("copy, compact and a shared eviction under a capture")
    r = share.Rollouts(pg, 4, 60, 4, 20, 2, 64, 3)
    r.append(0, range(30))
    r.evict(0, range(0, 30, 2))
    r.append(1, range(10))
    r.fork(1, 2)
    q = r.randn(4, 4, 64).to(share.DEV)
    want = r.cache.decode(q)
    free = r.cache.bm.free_blocks()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for call in (lambda: r.cache.copy(0, 3), lambda: r.cache.compact(), lambda: r.cache.compact(0),
                     lambda: r.cache.evict(2, [5])):
            with pytest.raises(RuntimeError, match="capture"):
                call()
        got = r.cache.decode(q)
    assert r.cache.bm.free_blocks() == free
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    r.cache.copy(0, 3)
    r.held[3] = dict(r.held[0])
    r.evict(2, [5])
    assert r.cache.compact(0) > 0
    r.check_decode("later", q.cpu(), *r.cache.decode(q), 0.125)
