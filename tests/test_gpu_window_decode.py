"""The two ways a windowed decode finds the visible slots (MI355X): its waves pick them, or, under tables too wide for
that, a kernel lists them; and units that pick more than once.  Against plain attention in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2609_35750_amd import inputs
from tests import operators_ref as ref
from tests.gpu_helpers import announce, assert_close, assert_lse, to_f64
from tests.test_gpu_weights import DECODE_CASES, DEV, _cache, _dev, _within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pg():
    from paper_2609_35750_amd import paged

    return paged


def _check(pg, c, d, table, q, q_pos, window, sinks, seqs):
    S, D, block = q.shape[0], q.shape[2], c["block"]
    scale = 1.0 / math.sqrt(D)
    kw = dict(q_pos=torch.from_numpy(q_pos).to(DEV), window=window, sinks=sinks)
    w = d["weight"].clone()
    o, lse = pg.kvs_paged_decode_ex(q.to(DEV), d["k"], d["v"], d["slot_pos"], table, d["nblk"], scale, slot_weight=w, **kw)
    o2, lse2 = pg.kvs_paged_decode_ex(q.to(DEV), d["k"], d["v"], d["slot_pos"], table, d["nblk"], scale, **kw)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    k64, v64, q64 = ref.f64(c["k"]), ref.f64(c["v"]), ref.f64(q)
    got, want = to_f64(w), ref.f64(c["weight"])
    bound, seen, known = np.zeros_like(want), np.zeros(len(want), dtype=bool), np.zeros(len(want), dtype=bool)
    for s in range(S):
        slots = ref.visible(c["slot_pos"], c["table"][s], c["nblk"][s], block, c["nb"], q_pos[s], window, sinks)
        seen[slots] = True
        if s not in seqs:
            continue
        if not slots:
            assert (o[s] == 0).all() and torch.isneginf(lse[s]).all()
            continue
        ro, rl, x, err = ref.decode(q64[s], k64, v64, slots, block, scale)
        assert_close(f"O seq {s}", to_f64(o[s]), ro)
        assert_lse(f"seq {s}", to_f64(lse[s]), rl)
        want[slots] += x
        bound[slots] += err + ref.U32 * want[slots]
        known[slots] = True
    _within("entries", got[known], want[known], bound[known])
    assert torch.equal(w.cpu()[~torch.from_numpy(seen)], c["weight"][~torch.from_numpy(seen)])


@pytest.mark.parametrize("case", [c for c in DECODE_CASES if c[7]],
                         ids=lambda c: f"S{c[0]}_n{c[2]}_bs{c[3]}_H{c[4]}x{c[5]}_D{c[6]}_W{c[7]}_S{c[8]}")
def test_tables_much_wider_than_what_they_hold(pg, case):
    """Entries behind seq_blocks are not looked at, whatever they hold; the slots are listed first."""
    S, lo, hi, block, Hq, Hkv, D, window, sinks = case
    announce(f"decode_ex wide {case}")
    c = _cache(S, lo, hi, block, Hkv, D, 77 + S)
    d = _dev(c)
    width = (1 << 21) // block if S < 100 else 4096
    table = torch.full((S, width), 10 ** 9, dtype=torch.int32, device=DEV)
    table[:, :c["table"].shape[1]] = d["table"]
    rng = np.random.default_rng(S)
    q_pos = rng.integers(-1, 2 * hi, S).astype(np.int32)
    _check(pg, c, d, table, inputs.randn_bf16((S, Hq, D), 5), q_pos, window, sinks, range(min(S, 20)))


def test_units_of_more_tiles_than_a_wave_picks_at_a_time(pg):
    """Three sequences of 85 tiles in 16 units of 128 KV heads: runs of 17 tiles."""
    announce("decode_ex: picks twice")
    c = _cache(3, 2704, 2704, 16, 128, 64, 5)
    d = _dev(c)
    q_pos = np.array([2703, 5300, 2000], dtype=np.int32)
    _check(pg, c, d, d["table"], inputs.randn_bf16((3, 128, 64), 6), q_pos, 2600, 7, range(3))


@pytest.mark.parametrize("S,tiles,Hkv,D", [(40, 28, 16, 128), (300, 30, 4, 64), (2, 1, 1, 128)])
def test_sequences_that_share_their_blocks(pg, S, tiles, Hkv, D):
    """Tables over the same blocks, each in an order of its own: O and LSE (the weights are unspecified then)."""
    announce(f"decode_ex: shared blocks {S} {tiles} {Hkv} {D}")
    c = _cache(1, 32 * tiles, 32 * tiles, 8, Hkv, D, 3, extra=0)
    rng = np.random.default_rng(1)
    table = np.stack([rng.permutation(c["table"][0]) for _ in range(S)]).astype(np.int32)
    d = _dev(c)
    q, q_pos = inputs.randn_bf16((S, 2 * Hkv, D), 9), rng.integers(0, 32 * tiles, S).astype(np.int32)
    nblk = torch.full((S,), table.shape[1], dtype=torch.int32, device=DEV)
    o, lse = pg.kvs_paged_decode_ex(q.to(DEV), d["k"], d["v"], d["slot_pos"], torch.from_numpy(table).to(DEV), nblk,
                                    q_pos=torch.from_numpy(q_pos).to(DEV), window=500, sinks=3)
    torch.cuda.synchronize()
    k64, v64, q64 = ref.f64(c["k"]), ref.f64(c["v"]), ref.f64(q)
    for s in range(0, S, 7):
        slots = ref.visible(c["slot_pos"], table[s], table.shape[1], 8, c["nb"], q_pos[s], 500, 3)
        if not slots:
            assert (o[s] == 0).all() and torch.isneginf(lse[s]).all()
            continue
        ro, rl, _, _ = ref.decode(q64[s], k64, v64, slots, 8, 1.0 / math.sqrt(D))
        assert_close(f"O seq {s}", to_f64(o[s]), ro)
        assert_lse(f"seq {s}", to_f64(lse[s]), rl)
