"""Attention weights of keys whose columns take a workgroup many steps (MI355X): several 64-row steps of several q-heads an
item, classes that change from step to step, chunk borders inside windows and evicted spans.  A sample of the keys of every
trace against the plain 64-bit form."""
import math

import numpy as np
import pytest
import torch

from paper_2609_35750_amd import inputs
from tests import operators_ref as ref
from tests.gpu_helpers import announce, to_f64
from tests.test_gpu_weights import DEV, _within

pytestmark = pytest.mark.gpu

CASES = [
    # lengths, varlen, Hq, Hkv, D, window, sinks, evict, last_rows
    ([5000] * 3, False, 16, 4, 128, 0, 0, False, 0),
    ([5000] * 3, False, 16, 4, 128, 0, 0, True, 0),
    ([4097, 1, 3000, 0, 2500], True, 12, 4, 64, 0, 0, True, 0),
    ([4097, 1, 3000, 0, 2500], True, 12, 4, 64, 700, 5, True, 0),
    ([5000] * 3, False, 16, 4, 128, 1500, 300, False, 0),
    ([2100] * 8, False, 24, 8, 128, 0, 0, True, 1000),
    ([2100, 333, 2000, 1999, 2100, 64, 2100, 2100], True, 24, 8, 64, 900, 0, False, 1000),
    ([30000], False, 10, 2, 128, 0, 0, True, 0),
    ([30000], True, 10, 2, 64, 5000, 64, False, 0),
]


def _want(q, k, lse, scale, window, sinks, e, rows, keys):
    """Weights of the sampled keys of one trace (fp64) and the bound of an fp32 evaluation's error, as ref.key_weights."""
    L, Hq, D = q.shape
    G = Hq // k.shape[1]
    i, j = np.arange(L)[:, None], keys[None, :]
    see = j <= i
    if window:
        see &= (i - j < window) | (j < sinks)
    if e is not None:
        see &= i < np.asarray(e, dtype=np.int64)[None, keys]
    if rows:
        see[:max(0, L - rows)] = False
    w, err = np.zeros(len(keys)), np.zeros(len(keys))
    for h in range(Hq):
        kk = k[keys, h // G]
        p = np.where(see, np.exp(np.where(see, scale * (q[:, h] @ kk.T) - lse[h][:, None], 0.0)), 0.0)
        de = ref.score_error(q[:, h], kk, scale, lse[h] / math.log(2.0))
        w += p.sum(0)
        err += (p * np.expm1(math.log(2.0) * de)).sum(0)
    return w, err + see.sum(0) * Hq * ref.U32 * w + 1e-37


@pytest.mark.parametrize("case", CASES,
                         ids=lambda c: f"{len(c[0])}xL{c[0][0]}_{'var' if c[1] else 'fix'}_H{c[2]}x{c[3]}_D{c[4]}_W{c[5]}_e{int(c[7])}_R{c[8]}")
def test_long_columns_match_the_plain_form(case):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import kvs

    lengths, varlen, Hq, Hkv, D, window, sinks, evict, rows = case
    announce(f"key weights, long columns {case}")
    B, n, T, G = len(lengths), sum(lengths), max(lengths), Hq // Hkv
    # The call's partial sums, chunks x parts of a group's q-heads of them a KV head and token, are what its workspace
    # grows by beyond LSE: fewer than the counted rows' steps of 64, so chunks are longer than a step; no multiple of the
    # group's q-heads, so parts hold several.
    size = lambda h: kvs.lib.kvs_key_weights_workspace(B, n, T, h, Hkv, D, rows)  # noqa: E731
    up = lambda x: -(-x // 256) * 256  # noqa: E731
    left = size(Hq) - up(4 * n) - up(8 * (B + n // 64 + 2)) - up(4 * n * Hq)
    parts = round(left / (4 * n * Hkv))
    assert up(4 * n * Hkv * parts) == left and parts < -(-min(T, rows or T) // 64) and (parts % G or parts < G), (left, parts)
    q, k = inputs.randn_bf16((n, Hq, D), 21), inputs.randn_bf16((n, Hkv, D), 22)
    rng = np.random.default_rng(n)
    ev = np.concatenate([np.arange(L) + 1 + rng.integers(0, L + 1, L) // rng.integers(1, 40, L) for L in lengths if L]) \
        if evict else None
    scale = 1.0 / math.sqrt(D)
    cu = np.concatenate([[0], np.cumsum(lengths)])
    # any LSE will do: the weights are defined by the one that is given
    lse = (6.0 + 2.0 * rng.standard_normal((Hq, n))).astype(np.float32)
    dev = lambda x: x.to(DEV) if varlen else x.to(DEV).view(B, -1, x.shape[1], D)  # noqa: E731
    l = torch.from_numpy(lse).to(DEV)
    e = None if ev is None else torch.from_numpy(ev.astype(np.int32)).to(DEV)
    if not varlen:
        l = l.view(Hq, B, -1).transpose(0, 1).contiguous()
        e = None if e is None else e.view(B, -1)
    kw = {"cu_seqlens": torch.from_numpy(cu.astype(np.int32)).to(DEV), "max_seqlen": T} if varlen else {}
    args = dict(window=window or None, sinks=sinks, last_rows=rows or None, **kw)
    w = kvs.kvs_key_weights(dev(q), dev(k), l, e, **args)
    again = kvs.kvs_key_weights(dev(q), dev(k), l, e, **args)
    torch.cuda.synchronize()
    assert torch.equal(w, again)
    got, q64, k64, l64 = to_f64(w).reshape(-1), ref.f64(q), ref.f64(k), lse.astype(np.float64)
    for b, (a, z) in enumerate(zip(cu[:-1], cu[1:])):
        L = int(z - a)
        if L == 0 or (b > 2 and not varlen):
            continue
        edges = np.concatenate([[0, 63, 64, 255, 256, L - 1, sinks, window], np.arange(64, L, 64 * 7), np.arange(255, L, 256)])
        keys = np.unique(np.concatenate([edges, rng.integers(0, L, 60)]).clip(0, L - 1))
        want, bound = _want(q64[a:z], k64[a:z], l64[:, a:z], scale, window, sinks, None if ev is None else ev[a:z], rows, keys)
        _within(f"trace {b}, {len(keys)} keys", got[a + keys], want, bound)
        assert (got[a + keys][want == 0.0] == 0.0).all()


@pytest.mark.parametrize("case", CASES,
                         ids=lambda c: f"{len(c[0])}xL{c[0][0]}_{'var' if c[1] else 'fix'}_H{c[2]}x{c[3]}_D{c[4]}_W{c[5]}_e{int(c[7])}_R{c[8]}")
def test_long_columns_count_rows_exactly(case):
    """Scores of 0 with LSE 0 give weight 1, with LSE 200 none (2^-288 is 0 in fp32): every key's weight is the number of
    the first kind among the rows and q-heads that see it, a whole number below 2^24, with no rounding anywhere."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import kvs

    lengths, varlen, Hq, Hkv, D, window, sinks, evict, rows = case
    announce(f"key weights, counted rows {case}")
    B, n, T = len(lengths), sum(lengths), max(lengths)
    rng = np.random.default_rng(n + 1)
    ev = np.concatenate([np.arange(L) + 1 + rng.integers(0, L + 1, L) // rng.integers(1, 40, L) for L in lengths if L]) \
        if evict else None
    cu = np.concatenate([[0], np.cumsum(lengths)])
    one = rng.random((Hq, n)) < 0.5
    l = torch.from_numpy(np.where(one, 0.0, 200.0).astype(np.float32)).to(DEV)
    shape = (n,) if varlen else (B, T)
    q = torch.zeros(*shape, Hq, D, dtype=torch.bfloat16, device=DEV)
    k = inputs.randn_bf16((n, Hkv, D), 2).to(DEV).view(*shape, Hkv, D)
    e = None if ev is None else torch.from_numpy(ev.astype(np.int32)).to(DEV).view(shape)
    if not varlen:
        l = l.view(Hq, B, T).transpose(0, 1).contiguous()
    kw = {"cu_seqlens": torch.from_numpy(cu.astype(np.int32)).to(DEV), "max_seqlen": T} if varlen else {}
    w = kvs.kvs_key_weights(q, k, l, e, window=window or None, sinks=sinks, last_rows=rows or None, **kw)
    torch.cuda.synchronize()
    got = to_f64(w).reshape(-1)
    for a, z in zip(cu[:-1], cu[1:]):
        L = int(z - a)
        sums = np.concatenate([[0], np.cumsum(one[:, a:z].sum(0))])   # of the rows before each
        j = np.arange(L)
        end = np.full(L, L) if ev is None else np.minimum(ev[a:z], L)
        if window:
            end = np.where(j < sinks, end, np.minimum(end, j + window))
        start = np.minimum(np.maximum(j, L - rows if rows else 0), end)
        np.testing.assert_array_equal(got[a:z], (sums[end] - sums[start]).astype(np.float64))
