"""Guard bands around every buffer that the calls for windows, weights and evictions write (MI355X): outputs, weights,
caches, workspaces of exactly the queries' sizes (of misleading contents), through the C ABI, two calls of other shapes
sharing one workspace in turn.  No guard byte changes, and the results are those of ordinary allocations."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_helpers import announce
from tests.test_gpu_canary import Banded, _p, _stream
from tests.test_gpu_weights import DEV, _cache, _dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kvs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import kvs as k

    return k


def _banded(shape, dtype, fill=None):
    b = Banded(shape, dtype, torch.device(DEV))
    if fill is not None:
        b.t.copy_(fill)
    return b


def _space(n):
    return _banded((max(n, 1),), torch.uint8)


@pytest.mark.parametrize("lengths,Hq,Hkv,D,window,sinks,rows", [
    ([130, 1, 0, 517], 8, 2, 128, 60, 5, 0), ([333], 6, 3, 64, 1, 0, 17), ([64, 64, 65], 16, 1, 128, 1000, 70, 64)])
def test_traces(kvs, lengths, Hq, Hkv, D, window, sinks, rows):
    announce(f"guard bands: window attention and key weights {lengths}")
    L = kvs.lib
    n, B, T = sum(lengths), len(lengths), max(lengths)
    gen = torch.Generator(device=DEV).manual_seed(3)
    q, do = (torch.randn(n, Hq, D, generator=gen, device=DEV).bfloat16() for _ in range(2))
    k, v = (torch.randn(n, Hkv, D, generator=gen, device=DEV).bfloat16() for _ in range(2))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32), device=DEV)
    scale = 1.0 / math.sqrt(D)
    kw = dict(cu_seqlens=cu, max_seqlen=T)
    o2, lse2 = kvs.kvs_window_attn_fwd(q, k, v, window, sinks, **kw)
    g2 = kvs.kvs_window_attn_bwd(do, q, k, v, o2, lse2, window, sinks, **kw)
    w2 = kvs.kvs_key_weights(q, k, lse2, window=window, sinks=sinks, last_rows=rows or None, **kw)
    o, dq = (_banded(q.shape, torch.bfloat16) for _ in range(2))
    dk, dv = (_banded(k.shape, torch.bfloat16) for _ in range(2))
    lse, w = _banded((Hq, n), torch.float32), _banded((n,), torch.float32)
    nf, nb = (f(B, n, T, Hq, Hkv, D) for f in (L.kvs_window_attn_fwd_workspace, L.kvs_window_attn_bwd_workspace))
    nk = L.kvs_key_weights_workspace(B, n, T, Hq, Hkv, D, rows)
    sf, sb, sk = _space(nf), _space(nb), _space(nk)
    st = _stream()
    assert L.kvs_window_attn_fwd(_p(q), _p(k), _p(v), None, _p(cu), _p(o.t), _p(lse.t), B, n, T, Hq, Hkv, D, scale, window,
                                 sinks, _p(sf.t), nf, st) == 0
    assert L.kvs_window_attn_bwd(_p(do), _p(q), _p(k), _p(v), _p(o.t), _p(lse.t), None, _p(cu), _p(dq.t), _p(dk.t),
                                 _p(dv.t), B, n, T, Hq, Hkv, D, scale, window, sinks, _p(sb.t), nb, st) == 0
    assert L.kvs_key_weights(_p(q), _p(k), _p(lse.t), None, _p(cu), _p(w.t), B, n, T, Hq, Hkv, D, scale, window, sinks,
                             rows, _p(sk.t), nk, st) == 0
    torch.cuda.synchronize()
    assert all(b.guards_intact() for b in (o, lse, dq, dk, dv, w, sf, sb, sk))
    for b, want in zip((o, lse, dq, dk, dv, w), (o2, lse2, *g2, w2)):
        assert torch.equal(b.t, want)


@pytest.mark.parametrize("block", [1, 5, 16, 64])
def test_caches(kvs, block):
    from paper_2609_35750_amd import paged

    announce(f"guard bands: decode_ex, evictions, appends, block size {block}")
    L = kvs.lib
    st = _stream()
    for S, lo, hi, Hq, Hkv, D, window, sinks in ((3, 0, 90, 8, 2, 128, 20, 3), (5, 200, 1500, 4, 4, 64, 0, 0),
                                                 (2, 4000, 6000, 32, 1, 64, 3000, 10), (260, 1, 70, 2, 1, 128, 0, 0)):
        c = _cache(S, lo, hi, block, Hkv, D, 7 + S, spare=0, extra=0)
        d = _dev(c)
        nb, mb = c["nb"], c["table"].shape[1]
        q = torch.randn(S, Hq, D, device=DEV).bfloat16()
        q_pos = torch.full((S,), hi, dtype=torch.int32, device=DEV)
        kw = dict(q_pos=q_pos, window=window, sinks=sinks) if window else {}
        w2 = d["weight"].clone()
        o2, lse2 = paged.kvs_paged_decode_ex(q, d["k"], d["v"], d["slot_pos"], d["table"], d["nblk"], slot_weight=w2, **kw)
        o, lse = _banded((S, Hq, D), torch.bfloat16), _banded((S, Hq), torch.float32)
        w, pos = _banded(w2.shape, torch.float32, d["weight"]), _banded(d["slot_pos"].shape, torch.int32, d["slot_pos"])
        kc, vc = (_banded(x.shape, torch.bfloat16, x) for x in (d["k"], d["v"]))
        need = L.kvs_paged_decode_ex_workspace(S, Hq, Hkv, D, nb, mb, block, window, sinks, 1)
        ws = _space(need)
        for _ in range(2):       # the second call finds the first one's lists and scores
            w.t.copy_(d["weight"])
            assert L.kvs_paged_decode_ex(_p(q), _p(kc.t), _p(vc.t), _p(pos.t), _p(w.t), _p(d["table"]), _p(d["nblk"]),
                                         _p(q_pos), _p(o.t), _p(lse.t), S, Hq, Hkv, D, nb, block, mb, 1.0 / math.sqrt(D),
                                         window, sinks, _p(ws.t), need, st) == 0
            torch.cuda.synchronize()
            assert all(b.guards_intact() for b in (o, lse, w, pos, kc, vc, ws))
            assert torch.equal(o.t, o2) and torch.equal(lse.t, lse2) and torch.equal(w.t, w2)
        keep = torch.full((S,), lo // 2, dtype=torch.int32, device=DEV)
        most = max(1, mb * block // 2)
        pos2 = d["slot_pos"].clone()
        out2, n2 = paged.kvs_paged_evict_lowest(w2, pos2, d["table"], d["nblk"], keep, block, sinks=2, recent=5, max_out=most)
        out, cnt = _banded((S, most), torch.int32), _banded((S,), torch.int32)
        need = L.kvs_paged_evict_lowest_workspace(S, mb, block)
        ws = _space(need)
        assert L.kvs_paged_evict_lowest(_p(w.t), _p(pos.t), _p(d["table"]), _p(d["nblk"]), _p(keep), _p(out.t), _p(cnt.t),
                                        S, nb, block, mb, 2, 5, most, _p(ws.t), need, st) == 0
        torch.cuda.synchronize()
        assert all(b.guards_intact() for b in (out, cnt, w, pos, ws))
        assert torch.equal(out.t, out2) and torch.equal(cnt.t, n2) and torch.equal(pos.t, pos2)
        # appends with weights: slots at both ends of the cache, one outside it
        n = 3
        slots = torch.tensor([0, nb * block - 1, nb * block], dtype=torch.int32, device=DEV)
        new = torch.randn(2, n, Hkv, D, device=DEV).bfloat16()
        at, wn = torch.arange(n, dtype=torch.int32, device=DEV), torch.rand(n, device=DEV)
        for wnew, want in ((wn, wn[:2]), (None, torch.zeros(2, device=DEV))):
            assert L.kvs_paged_append_weighted(_p(new[0]), _p(new[1]), _p(wnew) if wnew is not None else None, _p(at),
                                               _p(slots), n, _p(kc.t), _p(vc.t), _p(pos.t), _p(w.t), nb, block, Hkv, D,
                                               st) == 0
            torch.cuda.synchronize()
            assert all(b.guards_intact() for b in (kc, vc, pos, w))
            assert torch.equal(w.t[slots[:2].long()], want) and torch.equal(pos.t[slots[:2].long()], at[:2])
