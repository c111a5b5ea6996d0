"""Copies and moves of cache slots (MI355X): bit for bit what indexing gives, nothing beside the destinations written."""
import numpy as np
import pytest
import torch

from tests.gpu_helpers import announce

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def pg():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import paged

    return paged


def _cache(nb, Hkv, bs, D, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    k, v = (torch.randint(-2 ** 15, 2 ** 15, (nb, Hkv, bs, D), generator=g, device=DEV, dtype=torch.int16) for _ in range(2))
    pos = torch.randint(-1, 1000, (nb * bs,), generator=g, device=DEV, dtype=torch.int32)
    w = torch.rand(nb * bs, generator=g, device=DEV)
    return k.view(torch.bfloat16), v.view(torch.bfloat16), pos, w     # any bits, NaN among them


def _want(src, dst, bs, k, v, pos, w, move):
    k, v, pos, w = (x.clone() for x in (k.view(torch.int16), v.view(torch.int16), pos, w))
    s, d = src.long(), dst.long()
    ok = (s >= 0) & (s < pos.numel()) & (d >= 0) & (d < pos.numel())
    s, d = s[ok], d[ok]
    for x in (k, v):
        x[d // bs, :, d % bs] = x[s // bs, :, s % bs]
    w[d] = w[s]
    pos[d] = pos[s]
    if move:
        pos[s] = -1
    return k, v, pos, w


@pytest.mark.parametrize("nb,Hkv,bs,D,n", [(4, 1, 1, 64, 1), (9, 2, 5, 64, 17), (40, 8, 16, 128, 300), (700, 3, 1, 128, 350),
                                           (30, 5, 64, 64, 900), (600, 8, 16, 128, 4500)])
@pytest.mark.parametrize("move", [False, True])
def test_copies(pg, nb, Hkv, bs, D, n, move):
    announce(f"paged copy {nb} {Hkv} {bs} {D} {n} move {move}")
    k, v, pos, w = _cache(nb, Hkv, bs, D, n)
    order = torch.from_numpy(np.random.default_rng(n).permutation(nb * bs).astype(np.int32))
    src, dst = order[:n].to(DEV), order[n:2 * n].to(DEV)
    src = src[:dst.numel()].contiguous()
    want = _want(src, dst, bs, k, v, pos, w, move)
    pg.kvs_paged_copy(src, dst, k, v, pos, w, move=move)
    for got, ref in zip((k.view(torch.int16), v.view(torch.int16), pos, w), want):
        assert torch.equal(got, ref)


def test_pairs_outside_the_cache_are_skipped(pg):
    announce("paged copy, slots outside the cache")
    nb, Hkv, bs, D = 6, 2, 4, 64
    k, v, pos, w = _cache(nb, Hkv, bs, D, 3)
    src = torch.tensor([0, -1, 24, 2, 2 ** 31 - 1, 5, -2 ** 31], dtype=torch.int32, device=DEV)
    dst = torch.tensor([8, 9, 10, -5, 11, 24, 12], dtype=torch.int32, device=DEV)
    want = _want(src, dst, bs, k, v, pos, w, True)
    pg.kvs_paged_copy(src, dst, k, v, pos, w, move=True)
    for got, ref in zip((k.view(torch.int16), v.view(torch.int16), pos, w), want):
        assert torch.equal(got, ref)


def test_layers_and_nothing(pg):
    """Without positions and weights only K and V change; an empty list changes nothing."""
    announce("paged copy of another layer")
    k, v, pos, w = _cache(12, 2, 4, 128, 5)
    src, dst = torch.arange(0, 20, dtype=torch.int32, device=DEV), torch.arange(20, 40, dtype=torch.int32, device=DEV)
    want = _want(src, dst, 4, k, v, pos, w, False)
    pg.kvs_paged_copy(src, dst, k, v)
    assert torch.equal(k.view(torch.int16), want[0]) and torch.equal(v.view(torch.int16), want[1])
    pg.kvs_paged_copy(src[:0], dst[:0], k, v, pos, w, move=True)
    assert torch.equal(k.view(torch.int16), want[0])
    with pytest.raises(ValueError):
        pg.kvs_paged_copy(src, dst[:3], k, v)
    with pytest.raises(ValueError):
        pg.kvs_paged_copy(src.long(), dst, k, v)
    with pytest.raises(ValueError):
        pg.kvs_paged_copy(src, dst, k, v, pos[:5].contiguous())
    with pytest.raises(pg.KvsError):
        pg.kvs_paged_copy(src, dst, k, v, move=True)


def test_on_another_stream_and_in_a_graph(pg):
    announce("paged copy in a graph")
    k, v, pos, w = _cache(40, 2, 16, 64, 9)
    src, dst = torch.arange(0, 200, dtype=torch.int32, device=DEV), torch.arange(300, 500, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pg.kvs_paged_copy(src, dst, k, v, pos, w)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pg.kvs_paged_copy(src, dst, k, v, pos, w)
    for seed in range(3):
        k2, v2, pos2, w2 = _cache(40, 2, 16, 64, 20 + seed)
        for a, b in ((k, k2), (v, v2), (pos, pos2), (w, w2)):
            a.copy_(b)
        want = _want(src, dst, 16, k, v, pos, w, False)
        g.replay()
        torch.cuda.synchronize()
        for got, ref in zip((k.view(torch.int16), v.view(torch.int16), pos, w), want):
            assert torch.equal(got, ref)
