"""Attention of query rows over the live entries of a cache in 64 bits, with how far a bf16 result may be off.

For one row with scores s_j (j of the entries it sees) the kernels form, in fp32,
p_j = exp(s_j - m) with m within a factor 2^8 of the row's maximum, l = sum p_j,
and o = (sum bf16(p_j) v_j) / l, rounded to bf16; parts of the entries may be summed
apart and joined in fp32.  What that adds to the exact result, u = 2^-24:
  the result's rounding                2^-8 |o| (half a step of bf16)
  the rounding of each p_j             2^-8 E, E = sum w_j |v_j|, w_j = p_j / l
  a score: a sum of D products of bf16 numbers, and its scaling and exponential
                                       d = u (D + 8) scale max_j sum_d |q_d k_jd| + 4 u (relative to p_j), so
                                       2 d E with l's own
  the sums over n entries in fp32, and the joins    2 (n + 16) u E, an upper bound for any order
LSE: d + (n + 16) u + 2^-22 |LSE|.
"""
import numpy as np
import torch

U = 2.0 ** -24


def attend(q, k, v, scale, see=None):
    """q [n, Hq, D], k, v [m, Hkv, D], see [n, m] (None: everything); any float type.

    Returns O [n, Hq, D], LSE [n, Hq] in 64 bits and how far a kernel's may be off."""
    q, k, v = (x.detach().cpu().double() for x in (q, k, v))
    n, Hq, D = q.shape
    m, Hkv, _ = k.shape
    G = Hq // Hkv
    o, lse = torch.zeros(n, Hq, D, dtype=torch.float64), torch.full((n, Hq), -np.inf, dtype=torch.float64)
    off_o, off_lse = torch.zeros_like(o), torch.zeros_like(lse)
    if m == 0:
        return o, lse, off_o, off_lse
    see = torch.ones(n, m, dtype=torch.bool) if see is None else see
    some = see.any(1)
    for h in range(Hq):
        kh, vh = k[:, h // G], v[:, h // G]
        s = (q[:, h] @ kh.t() * scale).masked_fill(~see, -np.inf)
        lse[:, h] = torch.logsumexp(s, 1)
        w = torch.exp(s - lse[:, h].clamp(min=-1e300)[:, None])
        o[:, h] = w @ vh
        E = w @ vh.abs()
        size = (q[:, h].abs() @ kh.abs().t()).masked_fill(~see, 0).amax(1)
        d = U * (D + 8) * scale * size + 4 * U
        cnt = see.sum(1).double()
        off_o[:, h] = 2.0 ** -8 * (o[:, h].abs() + E) + (2 * d + 2 * (cnt + 16) * U)[:, None] * E + 2.0 ** -16 * E
        off_lse[:, h] = d + (cnt + 16) * U + 2.0 ** -22 * lse[:, h].abs().nan_to_num(posinf=0)
    off_o[~some], off_lse[~some] = 0, 0
    return o, lse, off_o, off_lse


def check(name, o, lse, want):
    ro, rl, off_o, off_lse = want
    o, lse = o.detach().cpu().double(), lse.detach().cpu().double()
    none = torch.isneginf(rl)
    assert torch.isfinite(o).all(), f"{name}: O is not finite"
    assert torch.equal(none, torch.isneginf(lse)), f"{name}: rows without an entry"
    ratio = ((o - ro).abs() / off_o.clamp(min=1e-300))[(off_o > 0)]
    far = float(ratio.max()) if ratio.numel() else 0.0
    assert far <= 1, f"{name}: O is {far:.3f} times its bound off"
    assert (o[off_o == 0] == 0).all(), f"{name}: O of rows without an entry"
    d = (lse - rl).abs()[~none] / off_lse[~none]
    far_lse = float(d.max()) if d.numel() else 0.0
    assert far_lse <= 1, f"{name}: LSE is {far_lse:.3f} times its bound off"
    print(f"[parity] {name}: O {far:.3f}, LSE {far_lse:.3f} of the bound", flush=True)
