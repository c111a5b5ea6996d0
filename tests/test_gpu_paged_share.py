"""Sequences that share the beginning of their tables, and several new tokens a sequence (MI355X): the decode over shared
prefixes and the attention of new tokens over the cache, against 64-bit attention over what each token sees."""
import math

import numpy as np
import pytest
import torch

from tests import rows_ref as ref
from tests.gpu_helpers import announce

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def pg():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import paged

    return paged


class Rollouts:
    """A cache and what each sequence holds: position -> (k, v).  Slots without an entry hold NaN and infinities."""

    def __init__(self, pg, S, nb, bs, mb, Hkv, D, seed, weights=False):
        self.cache = pg.PagedKVCache(nb, bs, S, mb, Hkv, D, device=DEV, weights=weights)
        self.cache.k.fill_(float("nan"))
        self.cache.v.fill_(float("nan"))
        self.cache.v[::2] = float("inf")
        self.g = torch.Generator().manual_seed(seed)
        self.held = [{} for _ in range(S)]
        self.Hkv, self.D = Hkv, D

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.g).bfloat16()

    def append(self, s, positions):
        positions = [int(p) for p in positions]
        k, v = self.randn(len(positions), self.Hkv, self.D), self.randn(len(positions), self.Hkv, self.D)
        self.cache.append(s, positions, k.to(DEV), v.to(DEV))
        self.held[s].update({p: (a, b) for p, a, b in zip(positions, k, v)})

    def evict(self, s, positions):
        self.cache.evict(s, positions)
        for p in positions:
            del self.held[s][int(p)]

    def fork(self, a, b):
        self.cache.fork(a, b)
        self.held[b] = dict(self.held[a])

    def kv(self, s):
        pos = sorted(self.held[s])
        if not pos:
            z = torch.zeros(0, self.Hkv, self.D)
            return torch.zeros(0, dtype=torch.int64), z, z
        return torch.tensor(pos), *(torch.stack([self.held[s][p][i] for p in pos]) for i in range(2))

    def check_decode(self, name, q, o, lse, scale):
        for s in range(len(self.held)):
            _, k, v = self.kv(s)
            ref.check(f"{name} seq {s}", o[s:s + 1], lse[s:s + 1], ref.attend(q[s:s + 1], k, v, scale))

    def check_extend(self, name, q, o, lse, scale, lengths, positions, window=None, sinks=0):
        at = 0
        for s, n in enumerate(lengths):
            if n:
                pos, k, v = self.kv(s)
                i = torch.as_tensor(positions[at:at + n])[:, None]
                see = pos[None] <= i
                if window:
                    see &= (i - pos[None] < window) | (pos[None] < sinks)
                ref.check(f"{name} seq {s}", o[at:at + n], lse[at:at + n], ref.attend(q[at:at + n], k, v, scale, see))
            at += n


def _grouped(pg, groups, alone, Hkv, D, bs, seed):
    """groups: [(prefix, own entries of each member)]; alone: entries of sequences of their own.  Sequences are shuffled."""
    S = sum(len(m) for _, m in groups) + len(alone)
    order = np.random.default_rng(seed).permutation(S).tolist()
    total = sum(p + sum(m) for p, m in groups) + sum(alone)
    longest = max([p + max(m) for p, m in groups] + alone)
    r = Rollouts(pg, S, total // bs + 3 * S + 5, bs, longest // bs + 4, Hkv, D, seed)
    at = 0
    for p, own in groups:
        first = order[at]
        r.append(first, range(p))
        for s in order[at + 1:at + len(own)]:
            r.fork(first, s)
        for s, n in zip(order[at:], own):
            r.append(s, range(p, p + n))
        at += len(own)
    for n in alone:
        r.append(order[at], range(n))
        at += 1
    return r


DECODE = [
    # groups, alone, Hq, Hkv, D, block size
    ([(1, [0, 0])], [], 1, 1, 64, 1),
    ([(1, [1, 0, 3])], [0, 1, 2], 4, 4, 64, 16),
    ([(40, [3, 9, 1, 20])], [], 8, 2, 128, 16),
    ([(33, [0, 0, 7]), (64, [31, 33])], [65, 0], 6, 2, 64, 5),
    ([(700, [20, 100, 1, 64, 300])], [500], 16, 2, 128, 1),
    ([(200, [5] * 70)], [], 8, 1, 64, 16),                      # rows of several row blocks, the last one ragged
    ([(100, list(range(0, 40))), (17, [2, 3]), (300, [1, 1, 1])], [9], 20, 4, 128, 64),
    ([(2500, [10, 1300, 0])], [4000], 4, 4, 128, 16),           # one row a KV head and sequence; long runs
    ([(1025, [1023, 1024]), (1024, [1, 1025])], [1, 1023], 64, 1, 128, 16),
]


@pytest.mark.parametrize("case", DECODE, ids=lambda c: f"{'_'.join(f'{p}x{len(m)}' for p, m in c[0])}_H{c[2]}x{c[3]}_D{c[4]}_bs{c[5]}")
def test_decode_over_shared_prefixes(pg, case):
    groups, alone, Hq, Hkv, D, bs = case
    announce(f"decode_shared {groups} {alone} {Hq} {Hkv} {D} {bs}")
    r = _grouped(pg, groups, alone, Hkv, D, bs, len(alone) + Hq)
    assert len(r.cache.device_groups()[1]) == len(groups)
    q = r.randn(len(r.held), Hq, D)
    scale = 1.0 / math.sqrt(D)
    o, lse = r.cache.decode(q.to(DEV))
    r.check_decode("shared", q, o, lse, scale)
    # evictions: part of a shared block, a span of shared blocks, own entries; then the groups are others
    big = max(range(len(r.held)), key=lambda s: len(r.held[s]))
    have = sorted(r.held[big])
    r.evict(big, have[:1] + have[len(have) // 3: len(have) // 2])
    o, lse = r.cache.decode(q.to(DEV), softmax_scale=0.3)
    r.check_decode("shared, evicted", q, o, lse, 0.3)


def test_everything_is_shared_or_gone(pg):
    """Members without entries of their own, a group whose prefix is evicted by all, sequences without any entry."""
    announce("decode_shared, nothing of one's own")
    r = Rollouts(pg, 6, 60, 4, 10, 2, 64, 5)
    r.append(2, range(11))
    for s in (0, 4):
        r.fork(2, s)
    r.append(5, range(3))
    q = r.randn(6, 4, 64)
    o, lse = r.cache.decode(q.to(DEV))
    r.check_decode("all shared", q, o, lse, 0.125)
    for s in (0, 2, 4):
        r.evict(s, sorted(r.held[s]))
    o, lse = r.cache.decode(q.to(DEV))
    assert torch.isneginf(lse[[0, 1, 2, 3, 4]]).all() and (o[[0, 1, 2, 3, 4]] == 0).all()
    r.check_decode("all gone", q, o, lse, 0.125)


def test_a_last_block_of_dead_slots_in_a_prefix(pg):
    """A shared block some of whose entries were evicted before the fork: its dead slots hold NaN and infinities."""
    announce("decode_shared, dead slots of a prefix")
    r = Rollouts(pg, 3, 200, 16, 60, 2, 128, 6)
    r.append(0, range(300))
    r.evict(0, [p for p in range(300) if p % 3 == 0 or 100 <= p < 140])
    r.cache.v[(r.cache.slot_pos < 0).view(-1, 16)[:, None, :].expand(-1, 2, -1)] = float("inf")
    r.fork(0, 1)
    r.fork(0, 2)
    q = r.randn(3, 8, 128)
    o, lse = r.cache.decode(q.to(DEV))
    r.check_decode("dead slots", q, o, lse, 1 / math.sqrt(128))


def test_large_and_equal_scores(pg):
    """Scores far apart (the maximum comes last, and in another split than most entries), and all the same."""
    announce("decode_shared, large scores")
    for amp in (0.0, 40.0):
        r = _grouped(pg, [(900, [30, 70, 200])], [], 2, 64, 16, 11)
        q = (r.randn(3, 4, 64).float() * amp).bfloat16()
        o, lse = r.cache.decode(q.to(DEV))
        r.check_decode(f"amplitude {amp}", q, o, lse, 0.125)


EXTEND = [
    # entries in front, evicted ones, new tokens, Hq, Hkv, D, block size, window, sinks
    ([0], 0, [1], 1, 1, 64, 1, None, 0),
    ([0, 5, 0], 0, [3, 0, 0], 4, 2, 64, 16, None, 0),
    ([100, 0, 33, 7], 3, [1, 65, 4, 0], 8, 2, 128, 16, None, 0),
    ([100, 0, 33, 7], 3, [1, 65, 4, 0], 8, 2, 128, 16, 20, 3),
    ([700, 300], 50, [130, 1], 6, 2, 64, 5, None, 0),
    ([700, 300], 50, [130, 257], 12, 4, 128, 1, 64, 4),
    ([2000], 200, [300], 16, 1, 128, 16, None, 0),
    ([2100, 1, 1024, 1023], 100, [4, 4, 4, 4], 8, 8, 128, 64, None, 0),
    ([5000], 10, [2], 32, 2, 64, 16, 1, 0),
    ([3000, 4000], 10, [40, 600], 5, 1, 64, 16, 900, 1000),
    ([513], 0, [512], 64, 1, 128, 16, 1 << 30, 0),
]


@pytest.mark.parametrize("case", EXTEND, ids=lambda c: f"{'_'.join(map(str, c[0]))}_n{'_'.join(map(str, c[2]))}_H{c[3]}x{c[4]}_D{c[5]}_bs{c[6]}_W{c[7]}_S{c[8]}")
def test_new_tokens(pg, case):
    front, gone, new, Hq, Hkv, D, bs, window, sinks = case
    announce(f"extend {case}")
    S = len(front)
    r = Rollouts(pg, S, sum(front + new) // bs + 4 * S, bs, max(a + b for a, b in zip(front, new)) // bs + 3, Hkv, D, Hq)
    rng = np.random.default_rng(S)
    positions = []
    for s in range(S):
        r.append(s, range(front[s]))
        if gone and front[s] > gone:
            r.evict(s, rng.choice(front[s], gone, replace=False))
        skip = 2 * s                                     # positions need not be those of the entries' number
        p = list(range(front[s] + skip, front[s] + skip + new[s]))
        r.append(s, p)
        positions += p
    q = r.randn(sum(new), Hq, D)
    scale = 1.0 / math.sqrt(D)
    o, lse = r.cache.extend(q.to(DEV), positions, new, window=window, sinks=sinks)
    r.check_extend("extend", q, o, lse, scale, new, positions, window, sinks)
    # one token a sequence is the decode of it
    if all(n == 1 for n in new):
        o2, lse2 = r.cache.decode(q.to(DEV))
        ref.check("decode", o2, lse2, ref.attend(q, *r.kv(0)[1:], scale))


def test_tokens_that_see_nothing_and_tokens_of_no_sequence(pg):
    """Positions in front of every entry give O = 0, LSE = -inf; rows behind the last sequence stay as they were."""
    announce("extend, empty rows")
    r = Rollouts(pg, 2, 40, 16, 10, 2, 64, 3)
    r.append(0, range(10, 60))
    q = r.randn(8, 4, 64)
    pos = [9, 10, 3, 59, 5, 5, 70, 70]                   # sequence 0: 5 tokens, sequence 1: one, nobody's: two
    pos[5] = -7
    o = torch.full((8, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((8, 4), 7.0, device=DEV)
    table, nblk = r.cache.device_tables()
    cu = torch.tensor([0, 5, 6], dtype=torch.int32, device=DEV)
    pg.kvs_paged_extend(q.to(DEV), r.cache.k, r.cache.v, r.cache.slot_pos, table, nblk,
                        torch.tensor(pos, dtype=torch.int32, device=DEV), cu, out=o, lse=lse)
    r.check_extend("empty rows", q, o, lse, 0.125, [5, 1], pos)
    assert (o[5] == 0).all() and torch.isneginf(lse[5]).all()
    assert (o[6:] == 7).all() and (lse[6:] == 7).all()


def test_positions_out_of_order(pg):
    """Tokens in any order of their positions, the same position twice, entries in any order of theirs."""
    announce("extend, any order")
    r = Rollouts(pg, 1, 80, 16, 60, 1, 128, 4)
    rng = np.random.default_rng(0)
    for part in np.array_split(rng.permutation(500), 9):
        r.append(0, part)
    pos = rng.integers(0, 520, 150).tolist()
    q = r.randn(150, 3, 128)
    for window, sinks in ((None, 0), (60, 5)):
        o, lse = r.cache.extend(q.to(DEV), pos, [150], window=window, sinks=sinks)
        r.check_extend("any order", q, o, lse, 1 / math.sqrt(128), [150], pos, window, sinks)


def test_all_tokens_of_a_trace_are_the_forward(pg):
    """New tokens over an empty cache: what the trainer's window attention and eviction mask give for the trace."""
    from paper_2609_35750_amd import kvs

    announce("extend against the trainer's forward")
    T, Hq, Hkv, D = 700, 8, 2, 128
    r = Rollouts(pg, 1, 60, 16, 50, Hkv, D, 8)
    r.append(0, range(T))
    q = r.randn(T, Hq, D)
    _, k, v = r.kv(0)
    for window, sinks in ((None, 0), (100, 7)):
        o, lse = r.cache.extend(q.to(DEV), range(T), [T], window=window, sinks=sinks)
        o2, lse2 = kvs.window_attn(q.to(DEV)[None], k.to(DEV)[None], v.to(DEV)[None], window or T, sinks)
        r.check_extend("trace", q, o, lse, 1 / math.sqrt(D), [T], list(range(T)), window, sinks)
        assert (lse2[0].t() - lse).abs().max() < 1e-4
        assert (o2[0].float() - o.float()).abs().max() <= 2 ** -7 * o.float().abs().max()


def test_graphs_streams_and_shared_workspaces(pg):
    """Captured calls replayed between eager ones, two graphs, a side stream: every replay gives the eager result."""
    announce("decode_shared and extend in graphs")
    r = _grouped(pg, [(300, [20, 60, 5]), (90, [9, 9])], [40], 2, 128, 16, 21)
    S, D = 6, 128
    table, nblk = r.cache.device_tables()
    group, blocks = r.cache.device_groups()
    q = r.randn(S, 8, D).to(DEV)
    new = [3, 0, 2, 1, 1, 4]
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]).astype(np.int32), device=DEV)
    pos = torch.tensor([400] * sum(new), dtype=torch.int32, device=DEV)
    qe = r.randn(sum(new), 8, D).to(DEV)
    args = (r.cache.k, r.cache.v, r.cache.slot_pos, table, nblk)

    def both():
        return (*pg.kvs_paged_decode_shared(q, *args, group, blocks), *pg.kvs_paged_extend(qe, *args, pos, cu, window=100, sinks=2))

    both()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = both()
        graphs.append((g, outs))
    side = torch.cuda.Stream()
    for turn in range(4):
        q.copy_(r.randn(S, 8, D))
        qe.copy_(r.randn(sum(new), 8, D))
        want = both()
        for g, outs in graphs:
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(outs, want):
                assert torch.equal(a, b)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = both()
        torch.cuda.current_stream().wait_stream(side)
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    r.check_decode("graphs", q.cpu(), want[0], want[1], 1 / math.sqrt(D))


def test_inputs_the_host_cannot_see(pg):
    """Groups, prefixes, offsets and tables out of range: nothing outside the buffers is touched, and sequences that are
    described as they should be get their results."""
    announce("decode_shared and extend, malformed inputs")
    r = _grouped(pg, [(60, [20, 6, 5])], [40, 33], 2, 64, 16, 31)
    S = 5
    table, nblk = (x.clone() for x in r.cache.device_tables())
    group, blocks = r.cache.device_groups()
    q = r.randn(S, 4, 64)
    args = (r.cache.k, r.cache.v, r.cache.slot_pos)
    alone = [s for s in range(S) if group[s] < 0]
    members = [s for s in range(S) if group[s] >= 0]
    odd = group.clone()
    odd[alone[0]], odd[alone[1]] = 2 ** 31 - 1, -2 ** 31
    o, lse = pg.kvs_paged_decode_shared(q.to(DEV), *args, table, nblk, odd, blocks)
    r.check_decode("groups out of range", q, o, lse, 0.125)
    # prefixes longer than the tables, negative, of nobody
    for b in ([2 ** 31 - 1, 5, -3], [-9, 2 ** 30, 0]):
        pg.kvs_paged_decode_shared(q.to(DEV), *args, table, nblk, group, torch.tensor(b, dtype=torch.int32, device=DEV))
    # as above with zero blocks in common: every sequence by itself
    o, lse = pg.kvs_paged_decode_shared(q.to(DEV), *args, table, nblk, group, torch.zeros(1, dtype=torch.int32, device=DEV))
    r.check_decode("no blocks in common", q, o, lse, 0.125)
    # table entries outside the cache read nothing; block counts beyond the table are cut
    wide = torch.cat([table, torch.full_like(table, -1), torch.full_like(table, 2 ** 31 - 1)], 1).contiguous()
    o, lse = pg.kvs_paged_decode_shared(q.to(DEV), *args, wide, torch.where(nblk == nblk.max(), torch.full_like(nblk, 2 ** 31 - 1), nblk),
                                        group, blocks)
    full = [s for s in range(S) if nblk[s] < nblk.max()]
    for s in full:
        ref.check(f"wide table seq {s}", o[s:s + 1], lse[s:s + 1], ref.attend(q[s:s + 1], *r.kv(s)[1:], 0.125))
    assert members
    n = 40
    qe, pos = r.randn(n, 4, 64), torch.full((n,), 1000, dtype=torch.int32, device=DEV)
    for cu in ([0, n, 0, n, 0, n], [5, 3, 1, -4, 2 ** 31 - 1, -2 ** 31], [n + 5] * 6, [-1] * 6):
        pg.kvs_paged_extend(qe.to(DEV), *args, table, nblk, pos, torch.tensor(cu, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()


def test_refusals(pg):
    r = _grouped(pg, [(60, [20, 6])], [], 2, 64, 16, 41)
    table, nblk = r.cache.device_tables()
    group, blocks = r.cache.device_groups()
    c = r.cache
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device=DEV)
    pos, cu = torch.zeros(2, dtype=torch.int32, device=DEV), torch.tensor([0, 1, 2], dtype=torch.int32, device=DEV)
    sh = lambda q=q, t=table, n=nblk, g=group, b=blocks, **kw: pg.kvs_paged_decode_shared(q, c.k, c.v, c.slot_pos, t, n, g, b, **kw)  # noqa: E731
    ex = lambda q=q, t=table, n=nblk, p=pos, u=cu, **kw: pg.kvs_paged_extend(q, c.k, c.v, c.slot_pos, t, n, p, u, **kw)  # noqa: E731
    sh(), ex()
    for call in (lambda: sh(q=q.float()), lambda: sh(q=q[:1].contiguous()), lambda: sh(g=group[:1].contiguous()), lambda: sh(b=blocks[:0]),
                 lambda: sh(g=group.long()), lambda: sh(q=torch.zeros(2, 4, 128, dtype=torch.bfloat16, device=DEV)),
                 lambda: sh(out=torch.zeros(2, 4, 64, device=DEV)), lambda: sh(lse=torch.zeros(2, 3, device=DEV)),
                 lambda: sh(q=q.cpu()),
                 lambda: ex(p=pos[:1].contiguous()), lambda: ex(u=cu[:2].contiguous()), lambda: ex(window=0),
                 lambda: ex(window=-3), lambda: ex(p=pos.long()), lambda: ex(q=q.half())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        sh(q=torch.zeros(4, 2, 64, dtype=torch.bfloat16, device=DEV).transpose(0, 1))   # not contiguous
    with pytest.raises(pg.KvsError):
        ex(sinks=-1)
    with pytest.raises(pg.KvsError):
        sh(softmax_scale=0.0)
    with pytest.raises(ValueError):
        c.extend(q, [0, 1], [1, 2])
    with pytest.raises(ValueError):
        c.extend(q, [0, 1], [3, -1])
    w = pg.PagedKVCache(4, 4, 2, 4, 1, 64, device=DEV, weights=True)
    with pytest.raises(ValueError):
        w.fork(0, 1)


def test_empty_calls(pg):
    r = _grouped(pg, [(60, [20, 6])], [], 2, 64, 16, 41)
    o, lse = r.cache.extend(torch.zeros(0, 4, 64, dtype=torch.bfloat16, device=DEV), [], [0, 0])
    assert o.shape == (0, 4, 64) and lse.shape == (0, 4)
