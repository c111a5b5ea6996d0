"""Attention weights on the GPU (MI355X): of a trace's keys, and of a cache's entries as the decode adds them; the decode
under a window.  Against plain 64-bit forms, with bounds from the roundings an fp32 evaluation makes."""
import math

import numpy as np
import pytest
import torch

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


@pytest.fixture(scope="module")
def pg(kvs):
    from paper_2609_35750_amd import paged

    return paged


def _within(name, got, want, bound):
    ratio = float((np.abs(got - want) / bound).max()) if got.size else 0.0
    print(f"[weights] {name}: worst error / bound {ratio:.3f}", flush=True)
    assert np.all(np.isfinite(got)) and ratio <= 1.0, name


# ---------------------------------------------------------------- keys of traces
KEY_CASES = [
    # lengths, varlen, Hq, Hkv, D, window, sinks, evict, last_rows
    ([1], False, 4, 2, 128, 0, 0, False, 0),
    ([2], False, 2, 2, 64, 1, 0, False, 1),
    ([64], False, 4, 1, 128, 0, 0, False, 0),
    ([257], False, 8, 2, 128, 0, 0, True, 0),
    ([600], False, 6, 2, 64, 0, 0, True, 37),
    ([600], False, 8, 1, 128, 50, 3, True, 0),
    ([330, 330], False, 3, 3, 64, 100, 130, False, 64),
    ([0, 1, 65, 300, 0, 256], True, 16, 2, 128, 0, 0, True, 64),
    ([513, 2, 100], True, 5, 1, 64, 1, 1, False, 0),
    ([130], False, 64, 1, 64, 0, 0, False, 1 << 30),
]


@pytest.mark.parametrize("case", KEY_CASES, ids=lambda c: f"L{'-'.join(map(str, c[0]))}_H{c[2]}x{c[3]}_D{c[4]}_W{c[5]}_R{c[8]}")
def test_key_weights_match_the_plain_form(kvs, case):
    lengths, varlen, Hq, Hkv, D, window, sinks, evict, rows = case
    announce(f"key weights {case}")
    n = sum(lengths)
    q, k = inputs.randn_bf16((n, Hq, D), 21), inputs.randn_bf16((n, Hkv, D), 22)
    rng = np.random.default_rng(n)
    ev = np.concatenate([np.arange(L) + 1 + rng.integers(0, L + 1, L) for L in lengths if L]) if evict else None
    scale = 1.0 / math.sqrt(D)
    cu = np.concatenate([[0], np.cumsum(lengths)])
    q64, k64 = ref.f64(q), ref.f64(k)
    lse = np.zeros((Hq, n))
    for a, z in zip(cu[:-1], cu[1:]):
        see = ref.mask(z - a, window, sinks, None if ev is None else ev[a:z])
        for h in range(Hq):
            s = np.where(see, scale * (q64[a:z, h] @ k64[a:z, h // (Hq // Hkv)].T), -np.inf)
            lse[h, a:z] = np.log(np.exp(s).sum(1))
    lse32 = lse.astype(np.float32)       # what the kernel is given
    dev = lambda x: x.to(DEV) if varlen else x.to(DEV).view(len(lengths), -1, x.shape[1], D)  # noqa: E731
    l = torch.from_numpy(lse32).to(DEV)
    e = None if ev is None else torch.from_numpy(ev.astype(np.int32)).to(DEV)
    if not varlen:
        l = l.view(Hq, len(lengths), -1).transpose(0, 1).contiguous()
        e = None if e is None else e.view(len(lengths), -1)
    kw = {"cu_seqlens": torch.from_numpy(cu.astype(np.int32)).to(DEV), "max_seqlen": max(lengths)} if varlen else {}
    args = dict(window=window or None, sinks=sinks, last_rows=rows or None, **kw)
    w = kvs.kvs_key_weights(dev(q), dev(k), l, e, **args)
    again = kvs.kvs_key_weights(dev(q), dev(k), l, e, **args)
    torch.cuda.synchronize()
    assert torch.equal(w, again)
    got = to_f64(w).reshape(-1)
    for a, z in zip(cu[:-1], cu[1:]):
        want, bound = ref.key_weights(q64[a:z], k64[a:z], lse32[:, a:z].astype(np.float64), scale, window, sinks,
                                      None if ev is None else ev[a:z], rows)
        _within(f"keys {a}..{z}", got[a:z], want, bound)


def test_key_weights_ignore_what_no_counted_query_sees(kvs):
    """NaN in queries, LSE and keys that do not take part; tokens behind the last trace keep what W held."""
    announce("key weights: masked NaN")
    n, Hq, Hkv, D, rows = 300, 4, 2, 128, 40
    q, k = inputs.randn_bf16((n, Hq, D), 1).to(DEV), inputs.randn_bf16((n, Hkv, D), 2).to(DEV)
    cu = torch.tensor([0, 280], dtype=torch.int32, device=DEV)
    e = torch.full((n,), 2 ** 31 - 1, dtype=torch.int32, device=DEV)
    e[20:30] = 200                     # gone before the counted queries
    lse = torch.randn(Hq, n, device=DEV) + 5.0
    kw = dict(cu_seqlens=cu, max_seqlen=280, check_cu=False, last_rows=rows)
    want = kvs.kvs_key_weights(q, k, lse, e, **kw)
    q[:240], k[20:30], lse[:, :240] = float("nan"), float("nan"), float("nan")
    out = torch.full((n,), 7.0, device=DEV)
    kvs.kvs_key_weights(q, k, lse, e, out=out, **kw)
    torch.cuda.synchronize()
    assert torch.equal(out[:280], want[:280]) and (out[280:] == 7.0).all()
    assert (out[20:30] == 0.0).all() and (out[:20] > 0).all()
    # a NaN score of one query reaches the keys that query sees, and no others
    lse[:, 250] = float("nan")
    kvs.kvs_key_weights(q, k, lse, e, out=out, **kw)
    torch.cuda.synchronize()
    assert out[:20].isnan().all() and out[30:251].isnan().all()
    assert torch.isfinite(out[20:30]).all() and torch.isfinite(out[251:280]).all()


def test_key_weights_of_a_long_trace_sum_to_its_rows(kvs):
    """Every softmax row sums to 1: all weights of 40,001 tokens, cut into many chunks, add up to rows x heads."""
    announce("key weights L=40001")
    gen = torch.Generator(device=DEV).manual_seed(5)
    q = torch.randn(1, 40001, 8, 64, generator=gen, device=DEV).bfloat16()
    k, v = (torch.randn(1, 40001, 2, 64, generator=gen, device=DEV).bfloat16() for _ in range(2))
    e = torch.full((1, 40001), 2 ** 31 - 1, dtype=torch.int32, device=DEV)
    _, lse = kvs.kvs_evict_attn_fwd(q, k, v, e)
    w = kvs.kvs_key_weights(q, k, lse).double().sum().item()
    # every weight is off by its score errors (about 2^-24 (64 mag + ...), below 2^-15 at these magnitudes)
    assert abs(w / (40001 * 8) - 1.0) < 2.0 ** -15


# ---------------------------------------------------------------- decode
def _cache(S, lo, hi, block, Hkv, D, seed, holes=0.2, spare=2, order="random", extra=1):
    """A cache of S sequences with scattered dead slots: torch tensors, and the host's view."""
    rng = np.random.default_rng(seed)
    pos = []
    for s in range(S):
        n = int(rng.integers(lo, hi, endpoint=True))
        p = np.full(-(-n // block) * block, -1, dtype=np.int64)
        p[:n] = np.arange(n) * (1 + s % 2)            # positions with gaps in every other sequence
        p[:n][rng.random(n) < holes] = -1
        if order == "reversed":
            p[:n] = p[:n][::-1].copy()
        pos.append(p.reshape(-1, block))
    nblk = np.array([len(p) for p in pos], dtype=np.int32)
    nb = int(nblk.sum()) + spare
    ids = rng.permutation(nb)
    table = np.zeros((S, int(nblk.max()) + extra), dtype=np.int32)
    slot_pos = np.full((nb, block), -1, dtype=np.int32)
    at = 0
    for s, p in enumerate(pos):
        mine = ids[at:at + len(p)]
        at += len(p)
        table[s, :len(p)] = mine
        slot_pos[mine] = p
    gen = torch.Generator().manual_seed(seed)
    k, v = (torch.randn(nb, Hkv, block, D, generator=gen).bfloat16() for _ in range(2))
    weight = torch.rand(nb * block, generator=gen) * 4.0
    return dict(table=table, nblk=nblk, slot_pos=slot_pos.reshape(-1), k=k, v=v, weight=weight, nb=nb, block=block)


def _dev(c, **more):
    d = {n: torch.from_numpy(c[n]).to(DEV) if isinstance(c[n], np.ndarray) else c[n].to(DEV)
         for n in ("table", "nblk", "slot_pos", "k", "v", "weight")}
    return {**d, **more}


DECODE_CASES = [
    # S, lo, hi, block, Hq, Hkv, D, window, sinks
    (1, 1, 1, 16, 4, 4, 128, 0, 0),
    (3, 0, 40, 16, 8, 2, 128, 0, 0),
    (2, 300, 700, 1, 16, 1, 128, 0, 0),
    (5, 10, 333, 5, 6, 3, 64, 0, 0),
    (4, 100, 400, 64, 32, 1, 64, 0, 0),
    (2, 3000, 5000, 16, 8, 2, 128, 0, 0),
    (300, 1, 90, 16, 4, 2, 64, 0, 0),                   # more sequences than a wave adds up by itself
    (1, 2, 2, 16, 4, 4, 64, 1, 0),
    (3, 50, 200, 16, 8, 2, 128, 1, 3),
    (4, 200, 900, 5, 64, 4, 128, 33, 4),
    (3, 300, 900, 1, 12, 4, 64, 100, 40),
    (2, 6000, 9000, 16, 8, 2, 128, 700, 64),            # lists of several chunks
    (2, 100, 300, 64, 4, 2, 128, 1 << 30, 0),
    (270, 5, 70, 2, 2, 1, 64, 20, 1),
]


@pytest.mark.parametrize("case", DECODE_CASES, ids=lambda c: f"S{c[0]}_n{c[2]}_bs{c[3]}_H{c[4]}x{c[5]}_D{c[6]}_W{c[7]}_S{c[8]}")
@pytest.mark.parametrize("order", ["ascending", "reversed"])
def test_decode_with_window_and_weights(pg, case, order):
    S, lo, hi, block, Hq, Hkv, D, window, sinks = case
    announce(f"decode_ex {case} {order}")
    c = _cache(S, lo, hi, block, Hkv, D, 31 + S, order=order)
    rng = np.random.default_rng(S)
    # queries at, behind and before the newest position; some see nothing at all
    top = np.array([max([-1] + [int(p) for p in c["slot_pos"].reshape(-1, block)[c["table"][s, :c["nblk"][s]]].reshape(-1)])
                    for s in range(S)])
    q_pos = np.maximum(top + rng.integers(-5, 3, S), -1).astype(np.int32)
    q = inputs.randn_bf16((S, Hq, D), 99)
    d = _dev(c)
    scale = 1.0 / math.sqrt(D)
    kw = dict(q_pos=torch.from_numpy(q_pos).to(DEV), window=window, sinks=sinks) if window else {}
    base = d["weight"].clone()
    o, lse = pg.kvs_paged_decode_ex(q.to(DEV), d["k"], d["v"], d["slot_pos"], d["table"], d["nblk"], scale,
                                    slot_weight=d["weight"], **kw)
    # without weights: the same bits of O and LSE
    o2, lse2 = pg.kvs_paged_decode_ex(q.to(DEV), d["k"], d["v"], d["slot_pos"], d["table"], d["nblk"], scale, **kw)
    again = base.clone()
    pg.kvs_paged_decode_ex(q.to(DEV), d["k"], d["v"], d["slot_pos"], d["table"], d["nblk"], scale, slot_weight=again, **kw)
    if not window:
        o3, lse3 = pg.kvs_paged_decode(q.to(DEV), d["k"], d["v"], d["slot_pos"], d["table"], d["nblk"], scale)
        assert torch.equal(o, o3) and torch.equal(lse, lse3)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and torch.equal(d["weight"], again)
    k64, v64, q64 = ref.f64(c["k"]), ref.f64(c["v"]), ref.f64(q)
    got_w, want_w = to_f64(d["weight"]), ref.f64(c["weight"])
    bound, seen = np.zeros_like(want_w), np.zeros(len(want_w), dtype=bool)
    for s in range(S):
        slots = ref.visible(c["slot_pos"], c["table"][s], c["nblk"][s], block, c["nb"], q_pos[s], window, sinks)
        ro, rl, w, err = ref.decode(q64[s], k64, v64, slots, block, scale)
        if not slots:
            assert (o[s] == 0).all() and torch.isneginf(lse[s]).all()
            continue
        if s < 8:
            assert_close(f"O seq {s}", to_f64(o[s]), ro)
            assert_lse(f"seq {s}", to_f64(lse[s]), rl)
        want_w[slots] += w
        bound[slots] += err + ref.U32 * want_w[slots]
        seen[slots] = True
    _within("entries", got_w[seen], want_w[seen], bound[seen])
    assert torch.equal(d["weight"].cpu()[~torch.from_numpy(seen)], c["weight"][~torch.from_numpy(seen)])


def test_dead_slots_may_hold_anything(pg):
    """NaN and infinities in K, V and weights of slots without an entry, in blocks nobody lists and behind a table's
    end; table entries outside the cache count as evicted."""
    announce("decode_ex: dead slots hold NaN")
    c = _cache(3, 100, 300, 16, 2, 128, 8)
    q = inputs.randn_bf16((3, 8, 128), 4).to(DEV)
    d = _dev(c, q_pos=torch.full((3,), 10 ** 6, dtype=torch.int32, device=DEV))
    table = torch.cat([d["table"], torch.full((3, 1), 10 ** 9, dtype=torch.int32, device=DEV)], 1).contiguous()

    def run(k, v, table, nblk, **kw):
        w = d["weight"].clone()
        out = pg.kvs_paged_decode_ex(q, k, v, d["slot_pos"], table, nblk, slot_weight=w, **kw)
        plain = pg.kvs_paged_decode(q, k, v, d["slot_pos"], table, nblk) if not kw else out
        return [*out, w, *plain]
    dead = (d["slot_pos"] < 0).view(-1, 1, 16, 1)
    k2 = torch.where(dead, torch.full_like(d["k"], float("nan")), d["k"])
    v2 = torch.where(dead, torch.full_like(d["v"], float("inf")), d["v"])
    for kw in ({}, {"q_pos": d["q_pos"], "window": 10 ** 6, "sinks": 0}):
        want = run(d["k"], d["v"], d["table"], d["nblk"], **kw)
        for k, v, t in ((k2, v2, d["table"]), (k2, v2, table)):
            got = run(k, v, t, d["nblk"], **kw)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, got))
    # one bad page inside the table, and counts beyond the table's width
    bad = table.clone()
    bad[1, 2] = -7
    good = c["table"].copy()
    o, lse = pg.kvs_paged_decode_ex(q, k2, v2, d["slot_pos"], bad, d["nblk"], q_pos=d["q_pos"], window=10 ** 6)
    torch.cuda.synchronize()
    # (position 0 is 10^6 behind the query, just outside the window)
    slots = [s for s in ref.visible(c["slot_pos"], good[1], c["nblk"][1], 16, c["nb"], 10 ** 6, 10 ** 6)
             if s // 16 != good[1, 2]]
    ro, rl, _, _ = ref.decode(ref.f64(q[1]), ref.f64(c["k"]), ref.f64(c["v"]), slots, 16, 1.0 / math.sqrt(128))
    assert_close("bad page O", to_f64(o[1]), ro)
    assert_lse("bad page", to_f64(lse[1]), rl)


def test_one_entry_weight_is_one(pg):
    """A query that sees one entry gives it weight 1 from each q-head, exactly."""
    announce("decode_ex: one entry")
    c = _cache(2, 200, 200, 16, 2, 64, 3, holes=0.0)
    d = _dev(c)
    w = torch.zeros_like(d["weight"])
    q_pos = torch.tensor([7, 14], dtype=torch.int32, device=DEV)
    pg.kvs_paged_decode_ex(inputs.randn_bf16((2, 8, 64), 1).to(DEV), d["k"], d["v"], d["slot_pos"], d["table"], d["nblk"],
                           q_pos=q_pos, window=1, slot_weight=w)
    torch.cuda.synchronize()
    slot = [int(np.nonzero(c["slot_pos"].reshape(-1, 16)[c["table"][s]].reshape(-1) == p)[0][0]) for s, p in ((0, 7), (1, 14))]
    at = [c["table"][s][x // 16] * 16 + x % 16 for s, x in enumerate(slot)]
    # 8 heads of probability exp2(s - LSE) with LSE rounded: 8 within a few steps
    assert abs(w[at].cpu().double() - 8.0).max() < 8 * 40 * ref.U32 and int((w != 0).sum()) == 2


def test_graph_replays_of_the_windowed_weighted_decode(pg):
    announce("decode_ex graph replays")
    c = _cache(6, 200, 2500, 16, 2, 128, 12)
    d = _dev(c, q_pos=torch.full((6,), 3000, dtype=torch.int32, device=DEV))
    q = inputs.randn_bf16((6, 8, 128), 2).to(DEV)
    o, lse = torch.empty_like(q), torch.empty(6, 8, device=DEV)
    start, w = d["weight"].clone(), d["weight"].clone()
    for kw in ({}, {"q_pos": d["q_pos"], "window": 1500, "sinks": 5}):
        def step():
            pg.kvs_paged_decode_ex(q, d["k"], d["v"], d["slot_pos"], d["table"], d["nblk"], slot_weight=w, out=o, lse=lse, **kw)  # noqa: B023
        side = torch.cuda.Stream()
        w.copy_(start)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        want = [x.clone() for x in (o, lse, w)]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step()
        for _ in range(3):
            w.copy_(start)
            o.fill_(float("nan"))
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, (o, lse, w)))
