"""Guard bands around every buffer that the copies of slots, the decode over shared prefixes and the attention of new
tokens write (MI355X): outputs, caches and workspaces of exactly the queries' sizes, of misleading contents, through the C
ABI, calls of other shapes sharing one workspace in turn.  No guard byte changes, whatever the tables, groups and offsets
hold, and well-formed calls give the results of ordinary allocations."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_helpers import announce
from tests.test_gpu_canary import Banded, _p, _stream

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def paged():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import paged as p

    return p


def _banded(shape, dtype, fill=None):
    b = Banded(shape, dtype, torch.device(DEV))
    if fill is not None:
        b.t.copy_(fill)
    return b


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _case(S, groups, lo, hi, block, Hkv, D, seed):
    """Tables of S sequences of lo .. hi blocks, those of a group beginning alike; one slot in eight is empty."""
    rng = np.random.default_rng(seed)
    n = rng.integers(lo, hi, S, endpoint=True)
    mb = hi + 1
    nb = S * mb + 3
    table = rng.permutation(nb)[: S * mb].reshape(S, mb)
    group = rng.integers(-1, groups, S)
    common = np.zeros(groups, dtype=np.int64)
    for g in range(groups):
        of = np.flatnonzero(group == g)
        if len(of):
            common[g] = rng.integers(0, n[of].min() + 1)
            table[of, : common[g]] = table[of[0], : common[g]]
    pos = np.arange(nb * block) % 997
    pos[rng.random(nb * block) < 1 / 8] = -1
    gen = torch.Generator(device=DEV).manual_seed(seed)
    k, v = (torch.randn(nb, Hkv, block, D, generator=gen, device=DEV).bfloat16() for _ in range(2))
    return _i32(table), _i32(n), _i32(pos), _i32(group), _i32(common), k, v, nb, mb


SHAPES = [(4, 2, 1, 30, 16, 8, 2, 128), (1, 1, 3, 3, 1, 4, 4, 64), (40, 3, 0, 12, 5, 12, 1, 64), (70, 1, 2, 40, 16, 16, 2, 128),
          (300, 80, 0, 4, 8, 6, 2, 64)]


def test_attention(paged):
    L = paged.lib
    most = 0
    for S, G, lo, hi, bs, Hq, Hkv, D in SHAPES:
        most = max(most, L.kvs_paged_decode_shared_workspace(S, G, Hq, Hkv, D, hi + 1, bs),
                   L.kvs_paged_extend_workspace(S, 3 * S, Hq, Hkv, D, hi + 1, bs))
    one = _banded((most,), torch.uint8)                     # the calls' common workspace
    for i, (S, G, lo, hi, bs, Hq, Hkv, D) in enumerate(SHAPES):
        announce(f"guard bands: decode_shared and extend {SHAPES[i]}")
        table, nblk, pos, group, common, k, v, nb, mb = _case(S, G, lo, hi, bs, Hkv, D, i)
        rng = np.random.default_rng(i)
        new = rng.integers(0, 7, S)
        n = int(new.sum())
        cu, q_pos = _i32(np.concatenate([[0], np.cumsum(new)])), _i32(rng.integers(-2, 1000, n))
        q = torch.randn(S, Hq, D, device=DEV).bfloat16()
        qe = torch.randn(n, Hq, D, device=DEV).bfloat16()
        scale = 1 / math.sqrt(D)
        cache = (_p(k), _p(v), _p(pos), _p(table), _p(nblk))
        for window, sinks in ((0, 0), (90, 3)):
            want = (*paged.kvs_paged_decode_shared(q, k, v, pos, table, nblk, group, common),
                    *paged.kvs_paged_extend(qe, k, v, pos, table, nblk, q_pos, cu, window=window or None, sinks=sinks))
            nd = L.kvs_paged_decode_shared_workspace(S, G, Hq, Hkv, D, mb, bs)
            ne = L.kvs_paged_extend_workspace(S, n, Hq, Hkv, D, mb, bs)
            for fill in (0xFF, 0x7F, None):
                sd, se = (_banded((x,), torch.uint8) for x in (nd, ne))
                if fill is None:
                    sd = se = one
                else:
                    sd.t.fill_(fill)
                    se.t.fill_(fill)
                o, lse = _banded(q.shape, torch.bfloat16), _banded((S, Hq), torch.float32)
                oe, lsee = _banded(qe.shape, torch.bfloat16), _banded((n, Hq), torch.float32)
                assert L.kvs_paged_decode_shared(_p(q), *cache, _p(group), _p(common), _p(o.t), _p(lse.t), S, G, Hq, Hkv, D,
                                                 nb, bs, mb, scale, _p(sd.t), nd, _stream()) == 0
                assert L.kvs_paged_extend(_p(qe), *cache, _p(q_pos), _p(cu), _p(oe.t), _p(lsee.t), S, n, Hq, Hkv, D, nb, bs,
                                          mb, scale, window, sinks, _p(se.t), ne, _stream()) == 0
                torch.cuda.synchronize()
                assert all(b.guards_intact() for b in (sd, se, o, lse, oe, lsee))
                for a, b in zip((o.t, lse.t, oe.t, lsee.t), want):
                    assert torch.equal(a, b)
        # anything in the tables, the groups and the offsets
        wild = lambda shape: _i32(rng.choice(np.array([-2 ** 31, -1, 0, 1, 2, 5, nb - 1, nb, 2 ** 31 - 1]), shape))  # noqa: E731
        for _ in range(4):
            t, b, g, c, u, p = wild((S, mb)), wild(S), wild(S), wild(G), wild(S + 1), wild(n)
            sd, se = (_banded((x,), torch.uint8) for x in (nd, ne))
            o, lse = _banded(q.shape, torch.bfloat16), _banded((S, Hq), torch.float32)
            oe, lsee = _banded(qe.shape, torch.bfloat16), _banded((n, Hq), torch.float32)
            for tab, blk, grp, com, cus, at in ((t, b, g, c, u, p), (table, nblk, g, c, u, p), (t, nblk, group, common, cu, q_pos),
                                                (table, b, group, c, cu, p)):
                assert L.kvs_paged_decode_shared(_p(q), _p(k), _p(v), _p(pos), _p(tab), _p(blk), _p(grp), _p(com), _p(o.t),
                                                 _p(lse.t), S, G, Hq, Hkv, D, nb, bs, mb, scale, _p(sd.t), nd, _stream()) == 0
                assert L.kvs_paged_extend(_p(qe), _p(k), _p(v), _p(pos), _p(tab), _p(blk), _p(at), _p(cus), _p(oe.t),
                                          _p(lsee.t), S, n, Hq, Hkv, D, nb, bs, mb, scale, 70, 3, _p(se.t), ne, _stream()) == 0
            torch.cuda.synchronize()
            assert all(x.guards_intact() for x in (sd, se, o, lse, oe, lsee))


@pytest.mark.parametrize("nb,Hkv,bs,D", [(5, 1, 1, 64), (9, 3, 5, 128), (20, 8, 16, 128)])
def test_copies(paged, nb, Hkv, bs, D):
    announce(f"guard bands: copies of slots {nb} {Hkv} {bs} {D}")
    gen = torch.Generator(device=DEV).manual_seed(nb)
    k, v = (_banded((nb, Hkv, bs, D), torch.bfloat16, torch.randn(nb, Hkv, bs, D, generator=gen, device=DEV)) for _ in range(2))
    pos = _banded((nb * bs,), torch.int32, torch.arange(nb * bs, dtype=torch.int32, device=DEV))
    w = _banded((nb * bs,), torch.float32, torch.rand(nb * bs, generator=gen, device=DEV))
    last = nb * bs - 1
    src, dst = _i32([0, last, -1, nb * bs, 2 ** 31 - 1, 1]), _i32([last - 1, 2, 0, 0, 0, nb * bs])
    k0, v0 = k.t.clone(), v.t.clone()
    paged.kvs_paged_copy(src, dst, k.t, v.t, pos.t, w.t, move=True)
    torch.cuda.synchronize()
    assert all(b.guards_intact() for b in (k, v, pos, w))
    for x, x0 in ((k, k0), (v, v0)):
        want = x0.clone()
        want[(last - 1) // bs, :, (last - 1) % bs] = x0[0, :, 0]
        want[2 // bs, :, 2 % bs] = x0[last // bs, :, last % bs]
        assert torch.equal(x.t, want)
    assert pos.t[last - 1] == 0 and pos.t[2] == last and pos.t[0] == pos.t[last] == -1 and pos.t[1] == 1
