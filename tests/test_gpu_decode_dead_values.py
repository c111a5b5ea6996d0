"""What slots without an entry hold in V does not reach a decode (MI355X), in any of its units and for any of its ways to find
the visible slots; infinities of live entries reach the columns they stand in, and no others."""
import numpy as np
import pytest
import torch

from paper_2609_35750_amd import inputs
from tests.gpu_helpers import announce
from tests.test_gpu_weights import DEV, _cache, _dev

pytestmark = pytest.mark.gpu

CASES = [
    # S, lo, hi, block, Hq, Hkv, D, holes
    (1, 30, 30, 16, 4, 2, 128, 0.3),
    (1, 20000, 20000, 16, 8, 2, 128, 0.4),      # many units of one sequence
    (6, 500, 4000, 16, 8, 2, 64, 0.9),
    (5, 10, 900, 5, 6, 3, 64, 0.3),
    (4, 300, 1500, 1, 16, 1, 128, 0.5),
    (300, 1, 90, 16, 4, 2, 64, 0.3),
]


@pytest.fixture(scope="module")
def pg():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import paged

    return paged


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"S{c[0]}_n{c[2]}_bs{c[3]}_H{c[4]}x{c[5]}_D{c[6]}")
@pytest.mark.parametrize("mode", ["plain", "weights", "window", "listed"])
@pytest.mark.parametrize("part", [0.02, 1.0], ids=["some", "all"])
def test_dead_values_change_no_bit(pg, case, mode, part):
    S, lo, hi, block, Hq, Hkv, D, holes = case
    announce(f"decode, dead values {case} {mode} {part}")
    c = _cache(S, lo, hi, block, Hkv, D, 60 + S + block, holes=holes)
    d = _dev(c)
    rng = np.random.default_rng(S)
    q = inputs.randn_bf16((S, Hq, D), 8).to(DEV)
    q_pos = torch.full((S,), 3 * hi, dtype=torch.int32, device=DEV)
    table = d["table"]
    if mode == "listed":     # too wide for the waves to pick
        table = torch.full((S, (1 << 21) // block if S < 100 else 4096), -1, dtype=torch.int32, device=DEV)
        table[:, :d["table"].shape[1]] = d["table"]
    dead = torch.from_numpy((c["slot_pos"] < 0) & (rng.random(len(c["slot_pos"])) < part)).to(DEV).view(-1, 1, block, 1)
    odd = torch.from_numpy(rng.choice(np.array([np.nan, np.inf, -np.inf, 3e38], dtype=np.float32), d["v"].shape)).to(DEV)

    def run(v):
        if mode == "plain":
            return pg.kvs_paged_decode(q, d["k"], v, d["slot_pos"], table, d["nblk"])
        w = d["weight"].clone()
        kw = {} if mode == "weights" else dict(q_pos=q_pos, window=2 * hi, sinks=3)
        return (*pg.kvs_paged_decode_ex(q, d["k"], v, d["slot_pos"], table, d["nblk"], slot_weight=w, **kw), w)
    want = run(torch.where(d["slot_pos"].view(-1, 1, block, 1) < 0, torch.zeros_like(d["v"]), d["v"]))
    got = run(torch.where(dead, odd.bfloat16(), d["v"]))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and torch.isfinite(got[0]).all()


@pytest.mark.parametrize("mode", ["plain", "window", "listed"])
@pytest.mark.parametrize("D", [64, 128])
def test_live_infinities_stay_in_their_columns(pg, mode, D):
    """An infinity in one column of a live entry's V, and dead NaN beside it: that column is infinite in the heads of the
    KV head and sequence, every other value is what it was."""
    announce(f"decode, live infinities {mode} {D}")
    c = _cache(3, 20, 45, 16, 2, D, 4, holes=0.3)
    d = _dev(c)
    q = (inputs.randn_bf16((3, 8, D), 8) * 0.1).to(DEV)      # scores near each other: no weight rounds to 0
    q_pos = torch.full((3,), 100, dtype=torch.int32, device=DEV)
    table = d["table"]
    if mode == "listed":
        table = torch.full((3, 1 << 17), -1, dtype=torch.int32, device=DEV)
        table[:, :d["table"].shape[1]] = d["table"]
    v = torch.where(d["slot_pos"].view(-1, 1, 16, 1) < 0, torch.full_like(d["v"], float("nan")), d["v"])

    def run(v):
        if mode == "plain":
            return pg.kvs_paged_decode(q, d["k"], v, d["slot_pos"], table, d["nblk"])
        return pg.kvs_paged_decode_ex(q, d["k"], v, d["slot_pos"], table, d["nblk"], q_pos=q_pos, window=101)
    want, lse = run(v)
    block = int(c["table"][1, 0])
    row = int(np.nonzero(c["slot_pos"].reshape(-1, 16)[block] >= 0)[0][-1])
    v2 = v.clone()
    v2[block, 1, row, 5] = float("inf")
    got, lse2 = run(v2)
    torch.cuda.synchronize()
    assert torch.equal(lse, lse2) and torch.isfinite(want).all()
    assert torch.isposinf(got[1, 4:, 5]).all()
    got[1, 4:, 5] = want[1, 4:, 5]
    assert torch.equal(got, want)
