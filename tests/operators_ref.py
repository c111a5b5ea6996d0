"""Plain 64-bit forms of the window, weight and eviction operators (test infrastructure), from their definitions:

    window:  query i sees key j  iff  j <= i < e_j  and  (i - j < W  or  j < S)
    weights: W_j = sum_h sum_{i sees j} exp(s_ij^h - LSE_i^h)
    evict:   the live, unprotected entries of lowest weight, until `keep` are left
"""
import math

import numpy as np

U32 = 2.0 ** -24     # half a step of fp32, relative


def f64(x):
    if hasattr(x, "detach"):
        return x.detach().to("cpu").double().numpy()
    return np.asarray(x, dtype=np.float64)


def mask(L, window, sinks, e=None):
    i, j = np.arange(L)[:, None], np.arange(L)[None, :]
    see = j <= i
    if window:
        see &= (i - j < window) | (j < sinks)
    if e is not None:
        see &= i < np.asarray(e, dtype=np.int64)[None, :]
    return see


def until(L, window, sinks, e=None):
    """The eviction indices with which the eviction mask is the window's: one past the last query that sees each key."""
    if L == 0:
        return np.zeros(0, dtype=np.int64)
    see = mask(L, window, sinks, e)
    return np.where(see.any(0), L - np.argmax(see[::-1], axis=0), np.arange(L)).astype(np.int64)


def score_error(q, k, scale, l2):
    """Bound of the error of x * scale_log2 - lse_log2 in fp32 (log2 units), [rows, keys]: the products of bf16 values
    are exact and added in fp32 (D roundings of partial sums no larger than the sum of magnitudes); scale * log2 e is
    rounded twice, LSE * log2 e twice (constant and product), and one fma rounds the result; exp2 adds one step."""
    D = q.shape[1]
    mag = (np.abs(q) @ np.abs(k).T) * scale / math.log(2.0)
    return U32 * (D * mag + 3.0 * mag + 3.0 * np.abs(l2)[:, None] + 2.0)


def key_weights(q, k, lse, scale, window=0, sinks=0, e=None, last_rows=0):
    """One trace: q [L,Hq,D], k [L,Hkv,D], lse [Hq,L] (all fp64).  Returns W [L] and the bound of an fp32 evaluation's
    error: every exponential's, and the additions' (any order: at most as many roundings as terms)."""
    L, Hq, _ = q.shape
    G = Hq // k.shape[1]
    see = mask(L, window, sinks, e)
    if last_rows:
        see[:max(0, L - last_rows)] = False
    w, err, terms = np.zeros(L), np.zeros(L), see.sum(0) * Hq
    for h in range(Hq):
        s = scale * (q[:, h] @ k[:, h // G].T)
        l2 = lse[h] / math.log(2.0)
        p = np.where(see, np.exp(np.where(see, s, 0.0) - np.where(see.any(1), lse[h], 0.0)[:, None]), 0.0)
        de = score_error(q[:, h], k[:, h // G], scale, np.where(see.any(1), l2, 0.0))
        w += p.sum(0)
        err += (p * np.expm1(math.log(2.0) * de)).sum(0)
    return w, err + terms * U32 * w + 1e-37


def visible(slot_pos, table, nblk, block, num_blocks, q_pos=None, window=0, sinks=0):
    """Slots a sequence's query sees, in the table's order."""
    out = []
    for b in table[:max(0, min(int(nblk), len(table)))]:
        if 0 <= b < num_blocks:
            for r in range(block):
                p = int(slot_pos[b * block + r])
                if p >= 0 and (not window or (p <= q_pos and (q_pos - p < window or p < sinks))):
                    out.append(int(b) * block + r)
    return out


def decode(q, k, v, slots, block, scale):
    """One sequence: q [Hq,D]; k, v caches [num_blocks,Hkv,block,D]; returns O, LSE, the slots' weights and their bound."""
    Hq, D = q.shape
    Hkv = k.shape[1]
    o, lse = np.zeros((Hq, D)), np.full(Hq, -np.inf)
    w, err = np.zeros(len(slots)), np.zeros(len(slots))
    if not slots:
        return o, lse, w, err
    sl = np.asarray(slots)
    for h in range(Hq):
        kk, vv = (x[sl // block, h // (Hq // Hkv), sl % block] for x in (k, v))
        s = scale * (kk @ q[h])
        m = s.max()
        lse[h] = m + math.log(np.exp(s - m).sum())
        p = np.exp(s - lse[h])
        o[h] = p @ vv
        w += p
        de = score_error(q[h][None], kk, scale, np.array([lse[h] / math.log(2.0)]))[0]
        # LSE itself: exponentials and additions of as many terms, one log2 and the way to natural logs and back
        de_lse = de.max() + U32 * (len(sl) + 4.0 + 6.0 * abs(lse[h]) / math.log(2.0)) / math.log(2.0)
        err += p * np.expm1(math.log(2.0) * (de + de_lse))
    return o, lse, w, err + (Hq + 1) * U32 * w


def evict_lowest(weight, slot_pos, table, nblk, block, num_blocks, keep, sinks, recent, max_out):
    """Slots one sequence loses, in the table's order."""
    slots = visible(slot_pos, table, nblk, block, num_blocks)
    if not slots:
        return []
    last = max(int(slot_pos[s]) for s in slots)
    rank = lambda w: (1, 0.0) if math.isnan(w) else (0, float(w) + 0.0)  # noqa: E731  (NaN last, -0 like 0)
    free = [(rank(weight[s]), at) for at, s in enumerate(slots) if sinks <= slot_pos[s] <= last - recent]
    n = max(0, min(len(slots) - max(int(keep), 0), len(free), max_out))
    return [slots[at] for at in sorted(at for _, at in sorted(free)[:n])]
