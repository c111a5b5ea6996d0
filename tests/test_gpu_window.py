"""Attention under a sliding window with sinks on the GPU (MI355X): against the 64-bit oracle under the mask's eviction
indices, its gradients against differences of a plain 64-bit loss, and bit for bit against the eviction-masked kernels."""
import gc
import math

import numpy as np
import pytest
import torch

from oracle import attention as orc
from paper_2609_35750_amd import inputs
from tests import operators_ref as ref
from tests.gpu_helpers import announce, assert_close, assert_lse, to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def kvs():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import kvs as k

    return k


def _evict(L, seed):
    """Eviction indices of random lifetimes, a third of the keys never evicted."""
    rng = np.random.default_rng(seed)
    e = np.arange(L) + 1 + rng.integers(0, max(L, 1), L)
    return np.where(rng.random(L) < 0.3, 2 ** 31 - 1, e).astype(np.int64)


CASES = [
    # lengths, varlen, Hq, Hkv, D, window, sinks, evict
    ([1], False, 4, 2, 128, 1, 0, False),
    ([2], False, 4, 4, 64, 1, 1, True),
    ([65], False, 6, 2, 128, 1, 0, False),            # a query sees itself only
    ([300], False, 8, 2, 128, 33, 4, False),
    ([257], False, 3, 1, 64, 64, 100, True),          # sinks end inside a tile and are wider than the window
    ([200, 200], False, 8, 8, 128, 100, 0, True),
    ([129], False, 8, 1, 128, 1 << 30, 7, False),     # window wider than the trace: causal
    ([190], False, 5, 1, 64, 20, 1 << 30, False),     # nothing but sinks: causal
    ([0, 1, 63, 0, 64, 300, 0], True, 8, 2, 128, 40, 5, True),
    ([511, 3, 130], True, 64, 1, 64, 90, 16, False),  # groups of 64
    ([700], False, 4, 1, 128, 17, 300, True),         # more sink tiles than window tiles
    ([1500], False, 4, 2, 64, 130, 1, False),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"L{'-'.join(map(str, c[0]))}_H{c[2]}x{c[3]}_D{c[4]}_W{c[5]}_S{c[6]}")
def test_forward_and_gradients_match_the_oracle(kvs, case):
    lengths, varlen, Hq, Hkv, D, window, sinks, evict = case
    announce(f"window attention {case}")
    n = sum(lengths)
    q, do = inputs.randn_bf16((n, Hq, D), 11), inputs.randn_bf16((n, Hq, D), 14)
    k, v = inputs.randn_bf16((n, Hkv, D), 12), inputs.randn_bf16((n, Hkv, D), 13)
    ev = np.concatenate([_evict(L, 5 + i) for i, L in enumerate(lengths)]) if evict else None
    cu = np.concatenate([[0], np.cumsum(lengths)])
    u = np.concatenate([ref.until(L, window, sinks, None if ev is None else ev[a:a + L])
                        for a, L in zip(cu[:-1], lengths)])
    scale = 1.0 / math.sqrt(D)
    dev = lambda x: x.to(DEV) if varlen else x.to(DEV).view(len(lengths), -1, x.shape[1], D)  # noqa: E731
    e = None if ev is None else torch.from_numpy(ev.astype(np.int32)).to(DEV)
    if e is not None and not varlen:
        e = e.view(len(lengths), -1)
    kw = {"cu_seqlens": torch.from_numpy(cu.astype(np.int32)).to(DEV), "max_seqlen": max(lengths)} if varlen else {}
    leaves = [dev(x).requires_grad_(True) for x in (q, k, v)]
    o, lse = kvs.window_attn(*leaves, window, sinks, e, **kw)
    dq, dk, dv = torch.autograd.grad(o, leaves, dev(do))
    torch.cuda.synchronize()
    cus = cu if varlen or len(lengths) > 1 else None
    want = orc.backward(q, k, v, u, scale, do, cus)
    E = orc.dq_rounding_scale(q, k, v, u, scale, do, np.arange(n), cus)
    S = orc.dkdv_rounding_rss(q, k, v, u, scale, do, cus)
    got = lambda x: to_f64(x).reshape(-1, x.shape[-2], D)  # noqa: E731
    assert_close("O", got(o), want["O"])
    lse64 = to_f64(lse) if varlen else to_f64(lse.permute(1, 0, 2).reshape(Hq, n))
    assert_lse("window", lse64, want["LSE"])
    assert_close("dQ", got(dq), want["dq"], E)
    assert_close("dK", got(dk), want["dk"], S=S[0])
    assert_close("dV", got(dv), want["dv"], S=S[1])


def test_gradients_match_differences(kvs):
    """<gradient, direction> against central differences of the plain 64-bit loss sum(dO * O)."""
    L, Hq, Hkv, D, window, sinks = 96, 4, 2, 64, 20, 3
    announce("window attention, gradients against differences")
    x = {"q": inputs.randn_bf16((1, L, Hq, D), 1), "k": inputs.randn_bf16((1, L, Hkv, D), 2),
         "v": inputs.randn_bf16((1, L, Hkv, D), 3)}
    do = inputs.randn_bf16((1, L, Hq, D), 4)
    see = torch.from_numpy(ref.mask(L, window, sinks))

    def loss(q, k, v):
        tot = 0.0
        for h in range(Hq):
            s = q[0, :, h] @ k[0, :, h // 2].T / math.sqrt(D)
            tot = tot + (do[0, :, h].double() * (torch.softmax(s.masked_fill(~see, -math.inf), 1) @ v[0, :, h // 2])).sum()
        return float(tot)
    leaves = {n: t.to(DEV).requires_grad_(True) for n, t in x.items()}
    o, _ = kvs.window_attn(leaves["q"], leaves["k"], leaves["v"], window, sinks)
    grads = dict(zip(leaves, torch.autograd.grad(o, list(leaves.values()), do.to(DEV))))
    base = {n: t.double() for n, t in x.items()}
    for n in x:
        g = grads[n].double().cpu()
        d = torch.randn(g.shape, generator=torch.Generator().manual_seed(9), dtype=torch.float64)
        eps = 1e-4
        up, dn = (loss(**{**base, n: base[n] + s * eps * d}) for s in (1, -1))
        diff = (up - dn) / (2 * eps)
        # the gradient's elements are rounded to bf16 (2^-8 each) after products of bf16-rounded P and dS (2^-8 each):
        # independent relative errors of about 2^-8 sqrt(3) of elements whose products with d add with random signs;
        # 8 times the root sum of squares covers it except with probability 1e-13
        room = 8.0 * 2.0 ** -8 * math.sqrt(3.0) * float((g * d).norm()) + 1e-5 * abs(diff)
        print(f"[diff] {n}: {float((g * d).sum()):.6f} against {diff:.6f}, room {room:.4f}", flush=True)
        assert abs(float((g * d).sum()) - diff) <= room


@pytest.mark.parametrize("shape", [(1, 4500, 8, 2, 128), (2, 2049, 6, 3, 64), (1, 20000, 4, 4, 128)], ids=str)
@pytest.mark.parametrize("window,sinks", [(1, 0), (100, 4), (1000, 65), (5000, 0)])
def test_bitwise_like_the_eviction_mask(kvs, shape, window, sinks):
    """The window's eviction indices through the eviction-masked kernels: the same products in the same order, fully
    masked blocks left out on one side, so every output has the same bits."""
    B, T, Hq, Hkv, D = shape
    announce(f"window bitwise {shape} W={window} S={sinks}")
    gen = torch.Generator(device=DEV).manual_seed(7)
    rnd = lambda h: torch.randn(B, T, h, D, generator=gen, device=DEV).bfloat16()  # noqa: E731
    q, k, v, do = rnd(Hq), rnd(Hkv), rnd(Hkv), rnd(Hq)
    ev = torch.from_numpy(np.stack([_evict(T, b) for b in range(B)]).astype(np.int32)).to(DEV)
    j = torch.arange(T, device=DEV, dtype=torch.int64)
    u = torch.where(j < sinks, ev.long(), torch.minimum(ev.long(), j + window)).int()
    o, lse = kvs.kvs_window_attn_fwd(q, k, v, window, sinks, ev)
    grads = kvs.kvs_window_attn_bwd(do, q, k, v, o, lse, window, sinks, ev)
    o2, lse2 = kvs.kvs_evict_attn_fwd(q, k, v, u)
    grads2 = kvs.kvs_evict_attn_bwd(do, q, k, v, o2, lse2, u)
    torch.cuda.synchronize()
    assert torch.equal(lse, lse2)
    for name, a, b in zip(("O", "dQ", "dK", "dV"), (o, *grads), (o2, *grads2)):
        assert torch.equal(a, b), name     # values: a sum of masked products may be 0 or -0


def test_rows_behind_the_last_trace_are_left_alone(kvs):
    announce("window attention: tokens behind the last trace")
    n, Hq, Hkv, D = 200, 4, 2, 64
    q, k, v = (inputs.randn_bf16((n, h, D), 3 + h).to(DEV) for h in (Hq, Hkv, Hkv))
    cu = torch.tensor([0, 70, 150], dtype=torch.int32, device=DEV)
    o, lse = torch.full_like(q, 7.0), torch.full((Hq, n), 7.0, device=DEV)
    kvs.kvs_window_attn_fwd(q, k, v, 16, 2, cu_seqlens=cu, max_seqlen=80, out=o, lse=lse, check_cu=False)
    torch.cuda.synchronize()
    assert (o[150:] == 7.0).all() and (lse[:, 150:] == 7.0).all()
    assert torch.isfinite(o[:150].float()).all() and not (lse[:, :150] == 7.0).any()


def test_captured_and_replayed_on_another_stream(kvs):
    """Forward and backward captured into a graph; replays between eager work equal the eager call bit for bit."""
    announce("window attention graph replays")
    gen = torch.Generator(device=DEV).manual_seed(1)
    q, do = (torch.randn(1, 3000, 8, 128, generator=gen, device=DEV).bfloat16() for _ in range(2))
    k, v = (torch.randn(1, 3000, 2, 128, generator=gen, device=DEV).bfloat16() for _ in range(2))
    outs = [torch.empty_like(q), torch.empty(1, 8, 3000, device=DEV), torch.empty_like(q), torch.empty_like(k),
            torch.empty_like(v)]

    def step():
        kvs.kvs_window_attn_fwd(q, k, v, 256, 8, out=outs[0], lse=outs[1])
        kvs.kvs_window_attn_bwd(do, q, k, v, outs[0], outs[1], 256, 8, dq=outs[2], dk=outs[3], dv=outs[4])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    want = [x.clone() for x in outs]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(4):
        for x in outs:
            x.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_captured_backward_beside_an_eager_graph_of_the_same_leaves(kvs):
    """Refused while the eager graph lives, by the host; the same capture works once it is gone."""
    announce("window attention: captured backward, refused and not")
    gen = torch.Generator(device=DEV).manual_seed(1)
    leaf = lambda h: torch.randn(1, 70, h, 64, generator=gen, device=DEV).bfloat16().requires_grad_()  # noqa: E731
    q, k, v = leaf(4), leaf(2), leaf(2)
    do = torch.randn(1, 70, 4, 64, generator=gen, device=DEV).bfloat16()
    o, _ = kvs.window_attn(q, k, v, 16, 2)
    want = torch.autograd.grad(o, (q, k, v), do, retain_graph=True)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o2, _ = kvs.window_attn(q, k, v, 16, 2)
        with pytest.raises(RuntimeError, match="captured"):
            torch.autograd.grad(o2, (q, k, v), do)
    del o, o2, g
    gc.collect()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        o, _ = kvs.window_attn(q, k, v, 16, 2)
        got = torch.autograd.grad(o, (q, k, v), do)
    for _ in range(3):
        for x in got:
            x.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_second_derivatives_are_refused(kvs):
    announce("window attention: double backward")
    q, k, v = (torch.randn(1, 40, h, 64, device=DEV).bfloat16().requires_grad_() for h in (4, 2, 2))
    o, _ = kvs.window_attn(q, k, v, 8)
    dq, = torch.autograd.grad(o.float().square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        dq.float().sum().backward()


def test_keys_and_values_that_are_one_tensor(kvs):
    """Its gradient is the sum of both, and one leaf in all three places gets all three."""
    announce("window attention: shared inputs")
    gen = torch.Generator(device=DEV).manual_seed(3)
    x, do = (torch.randn(1, 90, 2, 64, generator=gen, device=DEV).bfloat16() for _ in range(2))
    a, b, c = (x.clone().requires_grad_() for _ in range(3))
    o, _ = kvs.window_attn(a, b, c, 20, 3)
    parts = torch.autograd.grad(o, (a, b, c), do)
    y = x.clone().requires_grad_()
    o2, _ = kvs.window_attn(y, y, y, 20, 3)
    got, = torch.autograd.grad(o2, y, do)
    torch.cuda.synchronize()
    assert torch.equal(o, o2)
    want = sum(p.double() for p in parts)
    # two additions in bf16, each half a step of a partial sum
    bound = 2.0 * 2.0 ** -8 * sum(p.double().abs() for p in parts)
    assert ((got.double() - want).abs() <= bound).all()
