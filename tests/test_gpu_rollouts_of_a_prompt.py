"""Rollouts of one prompt, served and trained (MI355X): the prompt's entries are cached once and shared, each rollout takes
its tokens in chunks and one at a time; the trainer packs [prompt][rollout 1][rollout 2]... as one trace in which a
rollout's keys are evicted at its end.  Both against separate 64-bit attention over [prompt][rollout]."""
import numpy as np
import pytest
import torch

from oracle import attention as orc
from tests import rows_ref as ref
from tests.gpu_helpers import announce, assert_close, assert_lse, to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import kvs, paged

    return kvs, paged


def _trace(prompt, lengths, Hq, Hkv, D, seed):
    """q, k, v, dO of the trace, its evict_at, and each rollout's [first, last) row."""
    g = torch.Generator().manual_seed(seed)
    T = prompt + sum(lengths)
    q, k, v, do = (torch.randn(T, h, D, generator=g).bfloat16() for h in (Hq, Hkv, Hkv, Hq))
    ends = prompt + np.cumsum(lengths)
    spans = list(zip([prompt, *ends[:-1]], ends))
    e = np.full(T, T, dtype=np.int32)
    for a, b in spans:
        e[a:b] = b
    return q, k, v, do, e, spans


def _apart(q, k, v, do, prompt, spans, scale):
    """O, LSE and the gradients of separate causal attention over [prompt][rollout] in 64 bits; the prompt's rows once."""
    q, k, v = (x.double().requires_grad_(True) for x in (q, k, v))
    G = q.shape[1] // k.shape[1]
    outs, lses = [], []
    for r, (a, b) in enumerate([(0, prompt)] + spans):
        rows = list(range(a, b))
        keys = rows if r == 0 else list(range(prompt)) + rows
        kk, vv = (x[keys].repeat_interleave(G, 1) for x in (k, v))
        s = torch.einsum("ihd,jhd->hij", q[rows], kk) * scale
        behind = torch.tensor(keys)[None] > torch.tensor(rows)[:, None]
        s = s.masked_fill(behind[None], -np.inf)
        outs.append(torch.einsum("hij,jhd->ihd", s.softmax(-1), vv))
        lses.append(torch.logsumexp(s, -1))
    o = torch.cat(outs)
    o.backward(do.double())
    return o.detach(), torch.cat(lses, 1).detach(), q.grad, k.grad, v.grad


CASES = [(100, [40, 1, 33, 70], 8, 2, 128), (257, [130, 129, 3], 4, 4, 64), (1, [5, 64, 31], 5, 1, 128), (300, [90], 6, 2, 64)]


@pytest.mark.parametrize("prompt,lengths,Hq,Hkv,D", CASES)
def test_training(lib, prompt, lengths, Hq, Hkv, D):
    kvs, _ = lib
    announce(f"prompt {prompt} rollouts {lengths} H={Hq}/{Hkv} D={D}")
    q, k, v, do, e, spans = _trace(prompt, lengths, Hq, Hkv, D, 3)
    scale, T = D ** -0.5, len(e)
    want = _apart(q, k, v, do, prompt, spans, scale)
    leaves = [x[None].to(DEV).requires_grad_(True) for x in (q, k, v)]
    o, lse = kvs.evict_attn(*leaves, torch.from_numpy(e)[None].to(DEV), scale)
    o.backward(do[None].to(DEV))
    assert_close("O", to_f64(o[0]), want[0].numpy())
    assert_lse("LSE", to_f64(lse).reshape(Hq, T), want[1].numpy())
    E = orc.dq_rounding_scale(q, k, v, e, scale, do, np.arange(T))
    S = orc.dkdv_rounding_rss(q, k, v, e, scale, do)
    assert_close("dQ", to_f64(leaves[0].grad[0]), want[2].numpy(), E=E)
    assert_close("dK", to_f64(leaves[1].grad[0]), want[3].numpy(), S=S[0])
    assert_close("dV", to_f64(leaves[2].grad[0]), want[4].numpy(), S=S[1])


@pytest.mark.parametrize("block", [1, 16])
@pytest.mark.parametrize("prompt,lengths,Hq,Hkv,D", CASES)
def test_serving(lib, prompt, lengths, Hq, Hkv, D, block):
    _, paged = lib
    announce(f"prompt {prompt} rollouts {lengths} H={Hq}/{Hkv} D={D} blocks of {block}")
    q, k, v, _, _, spans = _trace(prompt, lengths, Hq, Hkv, D, 3)
    scale, S = D ** -0.5, len(lengths)
    room = (prompt + max(lengths)) // block + 2
    cache = paged.PagedKVCache(room * (S + 1), block, S, room, Hkv, D, device=DEV)
    cache.append(0, range(prompt), k[:prompt].to(DEV), v[:prompt].to(DEV))
    o, lse = cache.extend(q[:prompt].to(DEV), range(prompt), [prompt] + [0] * (S - 1))
    causal = lambda n, m: torch.arange(m)[None] <= torch.arange(m - n, m)[:, None]  # noqa: E731
    ref.check("prompt", o, lse, ref.attend(q[:prompt], k[:prompt], v[:prompt], scale, causal(prompt, prompt)))
    for s in range(1, S):
        cache.fork(0, s)
    assert cache.bm.free_blocks() == room * (S + 1) - -(-prompt // block), "the prompt is held once"
    done = [0] * S
    for step in range(max(lengths)):
        if all(d == n for d, n in zip(done, lengths)):
            break
        # every other turn one token a sequence, else up to 32 of them
        new = [min(n - d, 1 if step % 2 else 32) for d, n in zip(done, lengths)]
        rows, at = [], []
        for s, ((a, _), n) in enumerate(zip(spans, new)):
            i = a + done[s] + np.arange(n)
            pos = prompt + done[s] + np.arange(n)
            cache.append(s, pos, k[i].to(DEV), v[i].to(DEV))
            rows += i.tolist()
            at += pos.tolist()
        o, lse = cache.extend(q[rows].to(DEV), at, new)
        t = 0
        for s, ((a, _), n) in enumerate(zip(spans, new)):
            done[s] += n
            if n:
                kk, vv = (torch.cat([x[:prompt], x[a:a + done[s]]]) for x in (k, v))
                ref.check(f"step {step} seq {s}", o[t:t + n], lse[t:t + n],
                          ref.attend(q[rows[t:t + n]], kk, vv, scale, causal(n, prompt + done[s])))
            t += n
    # a token that decodes behind the last one of each, by either call
    last = q[[b - 1 for _, b in spans]]
    results = {"decode": cache.decode(last.to(DEV))}
    if S > 1:
        results["shared"] = paged.kvs_paged_decode_shared(last.to(DEV), cache.k, cache.v, cache.slot_pos,
                                                          *cache.device_tables(), *cache.device_groups())
    for name, (o, lse) in results.items():
        for s, (a, b) in enumerate(spans):
            kk, vv = (torch.cat([x[:prompt], x[a:b]]) for x in (k, v))
            ref.check(f"{name} seq {s}", o[s:s + 1], lse[s:s + 1], ref.attend(last[s:s + 1], kk, vv, scale))
