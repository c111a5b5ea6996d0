"""The operators as a rollout uses them: prompts scored under a window, their keys' weights into the cache, decode steps
that add weights, evictions down to a budget, on a window layer and a full layer; each step against 64-bit arithmetic."""
import math

import numpy as np
import pytest
import torch

from paper_2609_35750_amd import inputs
from tests import operators_ref as ref
from tests.gpu_helpers import announce, assert_close, assert_lse, to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import kvs, paged

    return kvs, paged


@pytest.mark.parametrize("block", [1, 16])
def test_rollouts_within_a_budget(lib, block):
    kvs, paged = lib
    S, Hq, Hkv, D, steps, budget, sinks, recent, window = 3, 8, 2, 128, 60, 200, 4, 40, 90
    announce(f"rollouts within a budget, block size {block}")
    prompts = [260, 130, 301]
    total = [p + steps for p in prompts]
    q, k, v = ([inputs.randn_bf16((n, h, D), 50 + 10 * h + i) for i, n in enumerate(total)] for h in (Hq, Hkv, Hkv))
    scale = 1.0 / math.sqrt(D)
    cache = paged.PagedKVCache(3 * (400 // block + 2), block, S, 400 // block + 2, Hkv, D, device=DEV, weights=True)
    # the prompts in one packed pass: outputs, then what each key received from the last 64 queries
    cu = torch.tensor(np.concatenate([[0], np.cumsum(prompts)]).astype(np.int32), device=DEV)
    pack = lambda x: torch.cat([t[:p] for t, p in zip(x, prompts)]).to(DEV)  # noqa: E731
    Q, K, V = pack(q), pack(k), pack(v)
    kw = dict(cu_seqlens=cu, max_seqlen=max(prompts))
    _, lse = kvs.window_attn(Q, K, V, window, sinks, **kw)
    w0 = kvs.kvs_key_weights(Q, K, lse, window=window, sinks=sinks, last_rows=64, **kw)
    for s, p in enumerate(prompts):
        a = int(cu[s])
        cache.append(s, np.arange(p), K[a:a + p], V[a:a + p], weights=w0[a:a + p])
    lse64 = to_f64(lse)
    want, err, live = [], [], []
    for s, p in enumerate(prompts):
        a = int(cu[s])
        w, e = ref.key_weights(ref.f64(q[s][:p]), ref.f64(k[s][:p]), lse64[:, a:a + p], scale, window, sinks, None, 64)
        want.append(dict(enumerate(w)))
        err.append(dict(enumerate(e)))
        live.append(list(range(p)))
    evicted = 0
    for t in range(steps):
        now = [p + t for p in prompts]
        for s in range(S):
            cache.append(s, [now[s]], k[s][now[s]:now[s] + 1].to(DEV), v[s][now[s]:now[s] + 1].to(DEV))
            live[s].append(now[s])
            want[s][now[s]] = err[s][now[s]] = 0.0
        Qt = torch.stack([q[s][now[s]] for s in range(S)]).to(DEV)
        o, l = cache.decode(Qt, accumulate=True)                                  # a full layer keeps the weights
        ow, lw = cache.decode(Qt, positions=now, window=window, sinks=sinks)      # a window layer over the same entries
        torch.cuda.synchronize()
        for s in range(S):
            see = [j for j in live[s] if now[s] - j < window or j < sinks]
            for name, at, oo, ll in (("full", live[s], o, l), ("window", see, ow, lw)):
                kk, vv = (ref.f64(x[s][at]).transpose(1, 0, 2)[None] for x in (k, v))       # as one block
                ro, rl, w, e = ref.decode(ref.f64(q[s][now[s]]), kk, vv, list(range(len(at))), len(at), scale)
                if t % 20 == 0 or t == steps - 1:
                    assert_close(f"{name} t={t} seq={s} O", to_f64(oo[s]), ro)
                    assert_lse(f"{name} t={t} seq={s}", to_f64(ll[s]), rl)
                if name == "full":
                    for j, x, y in zip(at, w, e):
                        want[s][j] += x
                        err[s][j] += y + ref.U32 * want[s][j]
        if t % 10 == 9:
            before = cache.slot_weight.cpu().numpy()
            slots = {}
            table, nblk = cache.bm.tables()
            pos = cache.slot_pos.cpu().numpy()
            for s in range(S):
                at = ref.visible(pos, table[s], nblk[s], block, cache.num_blocks)
                slots[s] = {int(pos[x]): x for x in at}
                assert sorted(slots[s]) == sorted(live[s])
                for j, x in slots[s].items():
                    assert abs(before[x] - want[s][j]) <= err[s][j] + 1e-30, (s, j)
            expect = [ref.evict_lowest(before, pos, table[s], nblk[s], block, cache.num_blocks, budget, sinks, recent, 10 ** 9)
                      for s in range(S)]
            gone = cache.evict_lowest(budget, sinks=sinks, recent=recent)
            for s in range(S):
                assert list(gone[s]) == [int(pos[x]) for x in expect[s]]
                live[s] = [j for j in live[s] if j not in set(gone[s].tolist())]
                assert cache.bm.live(s) == len(live[s]) == min(budget, len(live[s]) + len(gone[s]))
                evicted += len(gone[s])
    assert evicted > 150
    # released sequences leave nothing, and their slots start again at zero
    for s in range(S):
        cache.release(s)
    assert (cache.slot_pos == -1).all()
    cache.append(0, np.arange(50), k[0][:50].to(DEV), v[0][:50].to(DEV))
    got = cache.slot_weight[cache.slot_pos >= 0]
    assert got.numel() == 50 and (got == 0).all()


def test_weights_follow_scattered_slots(lib):
    """Entries appended in one call whose slots lie in more runs than a launch's arguments hold (device lists)."""
    _, paged = lib
    announce("append with weights over scattered slots")
    n = 1400
    cache = paged.PagedKVCache(2 * n, 1, 2, 2 * n, 1, 64, device=DEV, weights=True)
    kv = inputs.randn_bf16((2 * n, 1, 64), 3).to(DEV)
    cache.append(0, np.arange(2 * n), kv, kv)
    cache.evict(0, np.arange(0, 2 * n, 2))              # every other block is free
    w = torch.rand(n, device=DEV)
    slots = cache.append(1, np.arange(n), kv[:n], kv[n:], weights=w)
    torch.cuda.synchronize()
    assert np.abs(np.diff(slots)).min() >= 2
    assert torch.equal(cache.slot_weight[torch.from_numpy(slots).long().to(DEV)], w)
    at = torch.from_numpy(slots).long().to(DEV)
    assert torch.equal(cache.k[at, 0, 0], kv[:n, 0]) and torch.equal(cache.v[at, 0, 0], kv[n:, 0])
    assert torch.equal(cache.slot_pos[at].cpu(), torch.arange(n, dtype=torch.int32))
