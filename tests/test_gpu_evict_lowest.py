"""Eviction of the entries of lowest weight on the GPU (MI355X): exactly the plain form's entries, for every table shape."""
import numpy as np
import pytest
import torch

from tests import operators_ref as ref
from tests.gpu_helpers import announce
from tests.test_gpu_weights import DEV, _cache, _dev

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pg():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import paged

    return paged


def _weights(kind, n, rng):
    w = np.exp(2.0 * rng.standard_normal(n)).astype(np.float32)
    if kind == "ties":
        w = np.where(rng.random(n) < 0.5, np.float32(0.0), np.round(w).astype(np.float32))
    if kind == "odd":     # both zeros, both infinities, NaN, negative and tiny values
        w = rng.choice(np.array([0.0, -0.0, np.inf, -np.inf, np.nan, -1.0, 1e-40, -1e-40, 1.0, 3e38], dtype=np.float32), n)
    if kind == "equal":
        w[:] = 0.25
    return w


CASES = [
    # S, lo, hi, block, sinks, recent, extra table columns
    (1, 1, 1, 16, 0, 0, 0),
    (4, 0, 60, 16, 0, 0, 3),
    (3, 30, 90, 1, 2, 5, 0),
    (5, 500, 3000, 16, 4, 64, 1),
    (3, 3000, 9000, 5, 0, 100, 0),
    (2, 6000, 16000, 64, 64, 0, 0),
    (3, 2000, 5000, 1, 10, 500, 0),        # gathered first
    (2, 2000, 9000, 3, 0, 0, 0),
    (2, 20000, 40000, 16, 100, 1000, 5),   # gathered first, more places than a workgroup keeps
    (2, 17000, 30000, 1, 0, 7, 0),
    (70, 1, 200, 2, 1, 1, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"S{c[0]}_n{c[2]}_bs{c[3]}_sinks{c[4]}_recent{c[5]}")
@pytest.mark.parametrize("kind", ["spread", "ties", "odd", "equal"])
def test_exactly_the_lowest_leave(pg, case, kind):
    S, lo, hi, block, sinks, recent, extra = case
    announce(f"evict lowest {case} {kind}")
    c = _cache(S, lo, hi, block, 1, 64, 17 + S + block, extra=extra, order="reversed" if S == 5 else "ascending")
    rng = np.random.default_rng(S * 100 + block)
    c["weight"] = torch.from_numpy(_weights(kind, len(c["slot_pos"]), rng))
    live = [len(ref.visible(c["slot_pos"], c["table"][s], c["nblk"][s], block, c["nb"])) for s in range(S)]
    d = _dev(c)
    # keep: a part of each sequence; everything, nothing, more than there is, a negative number
    part = np.array([int(x * f) for x, f in zip(live, rng.random(S))], dtype=np.int32)
    some = np.array([[x, 0, x + 5, -3, x // 2][s % 5] for s, x in enumerate(live)], dtype=np.int32)
    for keep, most in ((part, None), (some, None), (part, 7), (np.zeros(S, dtype=np.int32), max(live + [1]))):
        slot_pos = d["slot_pos"].clone()
        w = d["weight"].clone()
        pos, counts = pg.kvs_paged_evict_lowest(w, slot_pos, d["table"], d["nblk"], torch.from_numpy(keep).to(DEV), block,
                                                sinks=sinks, recent=recent, max_out=most)
        torch.cuda.synchronize()
        want_pos, got = c["slot_pos"].copy(), pos.cpu().numpy()
        cap = got.shape[1]
        for s in range(S):
            gone = ref.evict_lowest(c["weight"].numpy(), c["slot_pos"], c["table"][s], c["nblk"][s], block, c["nb"],
                                    keep[s], sinks, recent, cap)
            assert int(counts[s]) == len(gone)
            np.testing.assert_array_equal(got[s, :len(gone)], c["slot_pos"][gone])
            assert (got[s, len(gone):] == -1).all()
            want_pos[gone] = -1
        np.testing.assert_array_equal(slot_pos.cpu().numpy(), want_pos)
        assert torch.equal(w.view(torch.int32), d["weight"].view(torch.int32))


def test_bad_tables_and_everything_protected(pg):
    """Table entries outside the cache hold nothing; with every entry protected none leaves."""
    announce("evict lowest: bad pages")
    c = _cache(3, 200, 400, 16, 1, 64, 5)
    d = _dev(c)
    bad = d["table"].clone()
    bad[0, 1], bad[2, 3] = 10 ** 9, -1
    host = bad.cpu().numpy()
    keep = torch.full((3,), 50, dtype=torch.int32, device=DEV)
    slot_pos = d["slot_pos"].clone()
    nblk = torch.tensor([c["nblk"][0], 0, c["nblk"][2]], dtype=torch.int32, device=DEV)
    pos, counts = pg.kvs_paged_evict_lowest(d["weight"], slot_pos, bad, nblk, keep, 16)
    torch.cuda.synchronize()
    for s in (0, 2):
        gone = ref.evict_lowest(c["weight"].numpy(), c["slot_pos"], host[s], c["nblk"][s], 16, c["nb"], 50, 0, 0, 10 ** 6)
        np.testing.assert_array_equal(pos[s, :int(counts[s])].cpu().numpy(), c["slot_pos"][gone])
    assert int(counts[1]) == 0
    for sinks, recent in ((10 ** 9, 0), (0, 10 ** 9), (100, 10 ** 6)):
        before = slot_pos.clone()
        _, counts = pg.kvs_paged_evict_lowest(d["weight"], slot_pos, d["table"], d["nblk"], torch.zeros_like(keep), 16,
                                              sinks=sinks, recent=recent)
        torch.cuda.synchronize()
        assert (counts == 0).all() and torch.equal(before, slot_pos)


@pytest.mark.parametrize("block", [1, 16])
def test_graph_replays(pg, block):
    announce(f"evict lowest graph replays bs={block}")
    c = _cache(4, 3000, 6000, block, 1, 64, 9)
    d = _dev(c)
    keep = torch.full((4,), 1000, dtype=torch.int32, device=DEV)
    slot_pos = d["slot_pos"].clone()
    want = [x.clone() for x in pg.kvs_paged_evict_lowest(d["weight"], slot_pos, d["table"], d["nblk"], keep, block, 4, 50)]
    marked = slot_pos.clone()
    g = torch.cuda.CUDAGraph()
    slot_pos.copy_(d["slot_pos"])
    with torch.cuda.graph(g):
        out = pg.kvs_paged_evict_lowest(d["weight"], slot_pos, d["table"], d["nblk"], keep, block, 4, 50)
    for _ in range(3):
        slot_pos.copy_(d["slot_pos"])
        out[0].fill_(5)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]) and torch.equal(slot_pos, marked)
