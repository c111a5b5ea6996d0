"""What O's rounding takes, kept by the windowed forward for its backward (MI355X): bit for bit where O is known exactly,
and gradients closer to the 64-bit ones."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_helpers import announce, to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def kvs():
    from paper_2609_35750_amd import kvs as k

    return k


def _expected(o32):
    """bf16 of fp32 values, and the eight bits below it."""
    bf = torch.from_numpy(o32).bfloat16()
    bits = bf.view(torch.int16).numpy().astype(np.int64) << 16
    d = (o32.view(np.int32).astype(np.int64) - bits + (1 << 31)) % (1 << 32) - (1 << 31)
    return bf, (np.minimum(d, 0x7FFF) >> 8).astype(np.int8)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("varlen", [False, True])
def test_remainders_of_means_of_two_values(kvs, D, varlen):
    """Queries of zero and a window of two: every score is 0 and every P 1, so O is the mean of two V, exact in fp32 and
    seldom in bf16.  (With other equal scores P, in bf16, and its sum, in fp32, are apart by a rounding.)"""
    announce(f"window remainders D={D} varlen={varlen}")
    L, Hq, Hkv = 333, 4, 2
    rng = np.random.default_rng(D)
    v = (rng.integers(-255, 256, (L, Hkv, D)) * 2.0 ** rng.integers(-3, 4, (L, Hkv, D))).astype(np.float32)
    k, q = rng.integers(-3, 4, (L, Hkv, D)).astype(np.float32), np.zeros((L, Hq, D), dtype=np.float32)
    cuts = [0, 100, 101, 300] if varlen else [0, L]
    want = np.zeros((L, Hq, D), dtype=np.float32)
    for a, b in zip(cuts, cuts[1:]):
        mean = v[a:b].copy()
        mean[1:] = (v[a:b][1:] + v[a:b][:-1]) * np.float32(0.5)
        want[a:b] = np.repeat(mean, Hq // Hkv, axis=1)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).bfloat16().to(DEV)[(...,) if varlen else None]  # noqa: E731
    kw = dict(cu_seqlens=torch.tensor(cuts, dtype=torch.int32, device=DEV), max_seqlen=199, check_cu=False) if varlen else {}
    Q, K, V = dev(q), dev(k), dev(v)
    rem = torch.full(Q.shape, 99, dtype=torch.int8, device=DEV)
    o, _ = kvs.kvs_window_attn_fwd(Q, K, V, 2, 0, rem=rem, **kw)
    plain, _ = kvs.kvs_window_attn_fwd(Q, K, V, 2, 0, **kw)
    torch.cuda.synchronize()
    n = cuts[-1]
    bf, bits = _expected(want)
    got = rem.reshape(L, Hq, D).cpu().numpy()
    assert torch.equal(o.reshape(L, Hq, D)[:n].cpu(), bf[:n]) and torch.equal(o.reshape(L, Hq, D)[:n], plain.reshape(L, Hq, D)[:n])
    np.testing.assert_array_equal(got[:n], bits[:n])
    assert (np.abs(bits[:n].astype(int)) > 16).mean() > 0.2 and (got[n:] == 99).all()


@pytest.mark.parametrize("L,D,W", [(300, 128, 16), (512, 64, 128)])
def test_gradients_are_closer_with_them(kvs, L, D, W):
    """dQ and dK against 64 bits, with the remainders (as window_attn takes them) and without."""
    announce(f"window remainders: gradients L={L} D={D} W={W}")
    H, S, scale = 4, 2, 1.0 / math.sqrt(D)
    gen = torch.Generator().manual_seed(L)
    q, k, v, do = (torch.randn(1, L, H, D, generator=gen).bfloat16() for _ in range(4))
    a, b, c, g = (x[0].transpose(0, 1).double() for x in (q, k, v, do))
    i, j = torch.arange(L)[:, None], torch.arange(L)[None, :]
    see = (j <= i) & ((i - j < W) | (j < S))
    p = torch.softmax((a @ b.transpose(1, 2) * scale).masked_fill(~see, -math.inf), -1)
    ds = p * (g @ c.transpose(1, 2) - (g * (p @ c)).sum(-1, keepdim=True))
    exact = (scale * ds @ b, scale * ds.transpose(1, 2) @ a)
    leaves = [x.to(DEV).requires_grad_() for x in (q, k, v)]
    o, lse = kvs.window_attn(*leaves, W, S)
    with_rem = torch.autograd.grad(o, leaves, do.to(DEV))
    without = kvs.kvs_window_attn_bwd(do.to(DEV), *(x.detach() for x in leaves), o.detach(), lse, W, S)
    torch.cuda.synchronize()
    assert torch.equal(with_rem[2], without[2])                        # dV takes no part
    far = lambda x, want: np.linalg.norm(to_f64(x)[0].transpose(1, 0, 2) - want.numpy())  # noqa: E731
    for x, y, want in zip(with_rem, without, exact):
        assert far(x, want) < 0.98 * far(y, want)
