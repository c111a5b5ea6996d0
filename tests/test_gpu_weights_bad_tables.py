"""Weights of a cache's entries under tables that list more entries outside the cache than in it (MI355X): an entry outside
counts as evicted, and every entry that exists gets its weight.  Against plain attention in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2609_35750_amd import inputs
from tests import operators_ref as ref
from tests.gpu_helpers import announce, assert_close, assert_lse, to_f64
from tests.test_gpu_weights import DEV, _cache, _dev, _within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pg():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import paged

    return paged


def _with_bad_entries(c, bad, front, rng):
    """The cache's tables with `bad` entries outside it a sequence, in front of the good ones or among them."""
    S = len(c["nblk"])
    table = np.zeros((S, int(c["nblk"].max()) + bad), dtype=np.int32)
    for s in range(S):
        n = int(c["nblk"][s])
        at = np.arange(bad, bad + n) if front else np.sort(rng.permutation(bad + n)[:n])
        row = rng.choice(np.array([-1, -7, c["nb"], 2 ** 31 - 1, 10 ** 9], dtype=np.int64), bad + n)
        row[at] = c["table"][s, :n]
        table[s, :bad + n] = row
    return table, (c["nblk"] + bad).astype(np.int32)


CASES = [
    # S, lo, hi, block, bad, front, Hq, Hkv, D, window, sinks
    (1, 64, 64, 16, 8, True, 4, 2, 128, 0, 0),
    (1, 64, 64, 16, 8, True, 4, 2, 128, 40, 3),
    (5, 100, 400, 16, 90, True, 8, 2, 128, 0, 0),
    (5, 100, 400, 16, 90, False, 6, 3, 64, 0, 0),
    (4, 50, 300, 1, 2000, False, 16, 1, 128, 0, 0),
    (4, 50, 300, 1, 2000, False, 12, 4, 64, 100, 5),
    (3, 90, 250, 5, 3000, True, 64, 64, 64, 0, 0),
    (300, 1, 90, 16, 20, False, 4, 2, 64, 0, 0),        # first tiles from a kernel of their own
    (270, 5, 70, 2, 100, False, 2, 1, 64, 20, 1),
    (2, 200, 500, 64, 9000, False, 8, 2, 128, 0, 0),
    (2, 200, 500, 64, 9000, False, 8, 2, 128, 300, 7),  # listed, not picked
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"S{c[0]}_bs{c[3]}_bad{c[4]}_H{c[6]}x{c[7]}_D{c[8]}_W{c[9]}")
def test_every_entry_gets_its_weight(pg, case):
    S, lo, hi, block, bad, front, Hq, Hkv, D, window, sinks = case
    announce(f"weights, bad entries {case}")
    c = _cache(S, lo, hi, block, Hkv, D, 51 + S + block, spare=0)
    rng = np.random.default_rng(S + block)
    table, nblk = _with_bad_entries(c, bad, front, rng)
    # more tiles are listed than the cache's slots make
    assert sum(-(-int(n) * block // 32) for n in nblk) > c["nb"] * block // 32 + S
    q = inputs.randn_bf16((S, Hq, D), 3)
    d = _dev({**c, "table": table, "nblk": nblk})
    scale = 1.0 / math.sqrt(D)
    q_pos = np.full(S, 2 * hi, dtype=np.int32) - (rng.integers(0, hi, S).astype(np.int32))
    kw = dict(q_pos=torch.from_numpy(q_pos).to(DEV), window=window, sinks=sinks) if window else {}
    args = (q.to(DEV), d["k"], d["v"], d["slot_pos"], d["table"], d["nblk"], scale)
    base = d["weight"].clone()
    o, lse = pg.kvs_paged_decode_ex(*args, slot_weight=d["weight"], **kw)
    again = base.clone()
    pg.kvs_paged_decode_ex(*args, slot_weight=again, **kw)
    o2, lse2 = pg.kvs_paged_decode_ex(*args, **kw)
    torch.cuda.synchronize()
    assert torch.equal(d["weight"], again) and torch.equal(o, o2) and torch.equal(lse, lse2)
    k64, v64, q64 = ref.f64(c["k"]), ref.f64(c["v"]), ref.f64(q)
    got, want = to_f64(d["weight"]), ref.f64(c["weight"])
    bound, seen = np.zeros_like(want), np.zeros(len(want), dtype=bool)
    for s in range(S):
        slots = ref.visible(c["slot_pos"], table[s], nblk[s], block, c["nb"], q_pos[s], window, sinks)
        if not slots:
            continue
        ro, rl, w, err = ref.decode(q64[s], k64, v64, slots, block, scale)
        if s < 8:
            assert_close(f"O seq {s}", to_f64(o[s]), ro)
            assert_lse(f"seq {s}", to_f64(lse[s]), rl)
        want[slots] += w
        bound[slots] += err + ref.U32 * want[slots]
        seen[slots] = True
    assert seen.any()
    _within("entries", got[seen], want[seen], bound[seen])
    assert torch.equal(d["weight"].cpu()[~torch.from_numpy(seen)], c["weight"][~torch.from_numpy(seen)])
