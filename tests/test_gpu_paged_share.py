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


def _decode(pg, r, q, scale=None):
    """The decode over shared prefixes, whatever the cache's own choice would be."""
    c = r.cache
    groups = c.device_groups()
    if not groups:
        groups = (torch.full((len(r.held),), -1, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV))
    return pg.kvs_paged_decode_shared(q.to(DEV), c.k, c.v, c.slot_pos, *c.device_tables(), *groups, scale)


def _grouped(pg, groups, alone, Hkv, D, bs, seed, room=0):
    """groups: [(prefix, own entries of each member)]; alone: entries of sequences of their own.  Sequences are shuffled.
    room: entries that any of them may take later."""
    S = sum(len(m) for _, m in groups) + len(alone)
    order = np.random.default_rng(seed).permutation(S).tolist()
    total = sum(p + sum(m) for p, m in groups) + sum(alone)
    longest = max([p + max(m) for p, m in groups] + alone)
    r = Rollouts(pg, S, total // bs + (3 + room // bs) * S + 5, bs, (longest + room) // bs + 4, Hkv, D, seed)
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
    ([(333, [7] * 13)], [50], 16, 2, 128, 16),                  # two row blocks of one wave's units
    ([(500, [40] * 9), (77, [1] * 11)], [], 20, 4, 64, 16),
    ([(90, [3] * 150)], [], 12, 6, 64, 8),                      # 300 rows
    ([(64, [2, 70]), (9, [1, 1, 5])], [300], 64, 1, 64, 16),    # 64 q-heads a KV head
]


@pytest.mark.parametrize("case", DECODE, ids=lambda c: f"{'_'.join(f'{p}x{len(m)}' for p, m in c[0])}_H{c[2]}x{c[3]}_D{c[4]}_bs{c[5]}")
def test_decode_over_shared_prefixes(pg, case):
    groups, alone, Hq, Hkv, D, bs = case
    announce(f"decode_shared {groups} {alone} {Hq} {Hkv} {D} {bs}")
    r = _grouped(pg, groups, alone, Hkv, D, bs, len(alone) + Hq)
    assert len(r.cache.device_groups()[1]) == len(groups)
    q = r.randn(len(r.held), Hq, D)
    scale = 1.0 / math.sqrt(D)
    o, lse = _decode(pg, r, q)
    r.check_decode("shared", q, o, lse, scale)
    o2, lse2 = r.cache.decode(q.to(DEV))          # by its own choice
    r.check_decode("decode", q, o2, lse2, scale)
    # evictions: part of a shared block, a span of shared blocks, own entries; then the groups are others
    big = max(range(len(r.held)), key=lambda s: len(r.held[s]))
    have = sorted(r.held[big])
    r.evict(big, have[:1] + have[len(have) // 3: len(have) // 2])
    o, lse = _decode(pg, r, q, 0.3)
    r.check_decode("shared, evicted", q, o, lse, 0.3)


def test_more_sequences_than_one_wave_plans(pg):
    """300 sequences in 90 groups, and 300 with new tokens."""
    announce("decode_shared and extend of 300 sequences")
    rng = np.random.default_rng(2)
    r = _grouped(pg, [(int(p), rng.integers(0, 30, 3).tolist()) for p in rng.integers(1, 60, 90)], rng.integers(0, 40, 30).tolist(),
                 2, 64, 8, 77, room=40)
    S = len(r.held)
    assert S == 300
    q = r.randn(S, 6, 64)
    o, lse = _decode(pg, r, q)
    r.check_decode("300 sequences", q, o, lse, 0.125)
    new = rng.choice([0, 1, 2, 40], S, p=[0.2, 0.5, 0.2, 0.1]).tolist()
    pos = []
    for s, n in enumerate(new):
        a = max(r.held[s], default=0) + 1
        r.append(s, range(a, a + n))
        pos += range(a, a + n)
    q = r.randn(len(pos), 6, 64)
    for window, sinks in ((None, 0), (20, 2)):
        o, lse = r.cache.extend(q.to(DEV), pos, new, window=window, sinks=sinks)
        r.check_extend("300 sequences", q, o, lse, 0.125, new, pos, window, sinks)


@pytest.mark.parametrize("Hkv,D,G,members", [(8, 128, 4, 40), (4, 64, 8, 3)])
def test_caches_beyond_4_gib(pg, Hkv, D, G, members):
    """K and V of 4.3 GB each: entries in the first and the last slots, for units of one wave and of four."""
    announce(f"decode_shared and extend in a large cache, {Hkv} {D}")
    bs = 16
    nb = (4300 << 20) // (bs * Hkv * D * 2)
    k, v = (torch.empty(nb, Hkv, bs, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    slot_pos = torch.full((nb * bs,), -1, dtype=torch.int32, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    blocks = torch.tensor([0, nb - 1, 1, nb - 2, nb // 2, nb - 3, nb - 4, 7], dtype=torch.int32, device=DEV)
    for x in (k, v):
        x[blocks.long()] = torch.randn(8, Hkv, bs, D, generator=g, device=DEV).bfloat16()
    slot_pos.view(nb, bs)[blocks.long()] = torch.arange(8 * bs, dtype=torch.int32, device=DEV).view(8, bs)
    S = members
    table = blocks.expand(S, 8).contiguous()
    nblk = torch.full((S,), 8, dtype=torch.int32, device=DEV)
    q = torch.randn(S, Hkv * G, D, generator=g, device=DEV).bfloat16()
    flat = [x[blocks.long()].transpose(1, 2).reshape(8 * bs, Hkv, D) for x in (k, v)]
    want = ref.attend(q, *flat, 1 / math.sqrt(D))
    o, lse = pg.kvs_paged_decode_shared(q, k, v, slot_pos, table, nblk, torch.zeros(S, dtype=torch.int32, device=DEV),
                                        torch.tensor([5], dtype=torch.int32, device=DEV))
    ref.check("shared", o, lse, want)
    one = torch.tensor([0, S], dtype=torch.int32, device=DEV)
    o, lse = pg.kvs_paged_extend(q, k, v, slot_pos, table[:1].contiguous(), nblk[:1].contiguous(),
                                 torch.full((S,), 1000, dtype=torch.int32, device=DEV), one)
    ref.check("extend", o, lse, want)
    src, dst = torch.arange(bs, dtype=torch.int32, device=DEV), (nb - 5) * bs + torch.arange(bs, dtype=torch.int32, device=DEV)
    pg.kvs_paged_copy(src, dst, k, v, slot_pos)
    assert torch.equal(k[nb - 5], k[0]) and torch.equal(v[nb - 5], v[0])


def test_everything_is_shared_or_gone(pg):
    """Members without entries of their own, a group whose prefix is evicted by all, sequences without any entry."""
    announce("decode_shared, nothing of one's own")
    r = Rollouts(pg, 6, 60, 4, 10, 2, 64, 5)
    r.append(2, range(11))
    for s in (0, 4):
        r.fork(2, s)
    r.append(5, range(3))
    q = r.randn(6, 4, 64)
    o, lse = _decode(pg, r, q)
    r.check_decode("all shared", q, o, lse, 0.125)
    for s in (0, 2, 4):
        r.evict(s, sorted(r.held[s]))
    o, lse = _decode(pg, r, q)
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
    o, lse = _decode(pg, r, q)
    r.check_decode("dead slots", q, o, lse, 1 / math.sqrt(128))


def test_large_and_equal_scores(pg):
    """Scores far apart (the maximum comes last, and in another split than most entries), and all the same."""
    announce("decode_shared, large scores")
    for amp in (0.0, 40.0):
        r = _grouped(pg, [(900, [30, 70, 200])], [], 2, 64, 16, 11)
        q = (r.randn(3, 4, 64).float() * amp).bfloat16()
        o, lse = _decode(pg, r, q)
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


@pytest.mark.parametrize("block", [1, 5, 16])
def test_life_of_two_groups(pg, block):
    """Rollouts of two prompts as an engine runs them: prompts, forks, chunks of observations, decode steps, spans evicted
    by some of the members, compaction, branches, releases; every output against what each sequence holds."""
    announce(f"life of two groups, block size {block}")
    Hq, Hkv, D, S, seed = 8, 2, 128, 8, 60 + block
    a = Rollouts(pg, S, 2000 // block + 60, block, 500 // block + 10, Hkv, D, seed)
    rng = np.random.default_rng(seed)
    scale = 1 / math.sqrt(D)
    nxt = [0] * S

    def chunk(lengths):
        pos = []
        for s, n in enumerate(lengths):
            p = list(range(nxt[s], nxt[s] + n))
            a.append(s, p)
            pos += p
            nxt[s] += n
        if pos:
            q = a.randn(len(pos), Hq, D)
            for window, sinks in ((None, 0), (50, 4)):
                o, lse = a.cache.extend(q.to(DEV), pos, lengths, window=window, sinks=sinks)
                a.check_extend("chunk", q, o, lse, scale, lengths, pos, window, sinks)

    def step():
        for s in range(S):
            if nxt[s]:
                a.append(s, [nxt[s]])
                nxt[s] += 1
        q = a.randn(S, Hq, D)
        o, lse = _decode(pg, a, q)
        a.check_decode("step", q, o, lse, scale)
        o2, lse2 = a.cache.decode(q.to(DEV))
        a.check_decode("step, plain", q, o2, lse2, scale)
        at = torch.tensor([max(n - 1, 0) for n in nxt], dtype=torch.int32, device=DEV)
        o3, lse3 = a.cache.decode(q.to(DEV), positions=at, window=40, sinks=3)
        for s in range(S):
            p, k, v = a.kv(s)
            see = ((int(at[s]) - p < 40) | (p < 3))[None]
            ref.check("step, window", o3[s:s + 1], lse3[s:s + 1], ref.attend(q[s:s + 1], k, v, scale, see))

    chunk([120, 0, 0, 0, 77, 0, 0, 0])
    for s in (1, 2, 3):
        a.fork(0, s)
        nxt[s] = nxt[0]
    for s in (5, 6):
        a.fork(4, s)
        nxt[s] = nxt[4]
    step()
    chunk([30, 1, 0, 64, 9, 33, 0, 0])
    step()
    a.evict(1, list(range(16, 48)))            # a span of the prompt, by one member
    a.evict(3, list(range(5, 9)) + [60])
    for s in (0, 4):
        a.evict(s, rng.choice(sorted(a.held[s])[-25:], 10, replace=False).tolist())
    step()
    before = [dict(h) for h in a.held]
    a.cache.compact()
    assert a.held == before
    step()
    a.cache.copy(1, 7)
    a.held[7], nxt[7] = dict(a.held[1]), nxt[1]
    step()
    a.cache.release(2)
    a.held[2], nxt[2] = {}, 0
    a.cache.release(4)
    a.held[4], nxt[4] = {}, 0
    step()
    a.fork(5, 4)
    nxt[4] = nxt[5]
    chunk([5, 0, 0, 12, 40, 40, 1, 3])
    for s in range(S):
        a.cache.release(s)
    assert a.cache.bm.free_blocks() == a.cache.num_blocks
    assert (a.cache.slot_pos == -1).all()


def test_copies_keep_weights(pg):
    """A cache that keeps weights: copies take them along, compaction too, and the eviction by them goes on as before."""
    announce("weights through copies and compaction")
    Hkv, D, bs = 2, 64, 8
    r = Rollouts(pg, 3, 60, bs, 30, Hkv, D, 71, weights=True)
    r.append(0, range(100))
    w = torch.rand(100)
    table, n = r.cache.bm.tables()
    slots = torch.from_numpy((table[0, :n[0], None] * bs + np.arange(bs)).reshape(-1)[:100]).long()
    r.cache.slot_weight[slots.to(DEV)] = w.to(DEV)
    r.cache.copy(0, 1)
    r.held[1] = dict(r.held[0])
    gone = np.random.default_rng(1).choice(100, 55, replace=False)
    r.evict(0, gone)
    r.evict(1, gone)
    assert r.cache.compact(0) > 0
    left = sorted(set(range(100)) - set(gone.tolist()))
    for s in (0, 1):
        table, n = r.cache.bm.tables()
        slots = torch.from_numpy((table[s, :n[s], None] * bs + np.arange(bs)).reshape(-1)).long()
        pos = r.cache.slot_pos.cpu()[slots]
        assert sorted(pos[pos >= 0].tolist()) == left
        assert torch.equal(r.cache.slot_weight.cpu()[slots][pos >= 0], w[pos[pos >= 0].long()])
    out = r.cache.evict_lowest(20)
    want = sorted(sorted(left, key=lambda p: float(w[p]))[: len(left) - 20])
    assert sorted(out[0].tolist()) == want and sorted(out[1].tolist()) == want


def test_two_streams_at_once(pg):
    """Calls on two streams at the same time, each with a workspace of its own."""
    announce("decode_shared and extend on two streams")
    r = _grouped(pg, [(400, [50, 60, 5, 1])], [200], 2, 128, 16, 81)
    table, nblk = r.cache.device_tables()
    group, blocks = r.cache.device_groups()
    args = (r.cache.k, r.cache.v, r.cache.slot_pos, table, nblk)
    q = r.randn(5, 16, 128).to(DEV)
    qe = r.randn(200, 16, 128).to(DEV)
    cu = torch.tensor([0, 90, 90, 200, 200, 200], dtype=torch.int32, device=DEV)
    pos = torch.full((200,), 1000, dtype=torch.int32, device=DEV)
    want = [x.clone() for x in (*pg.kvs_paged_decode_shared(q, *args, group, blocks), *pg.kvs_paged_extend(qe, *args, pos, cu))]
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    torch.cuda.synchronize()
    for _ in range(20):
        with torch.cuda.stream(streams[0]):
            got[0].append(pg.kvs_paged_decode_shared(q, *args, group, blocks))
        with torch.cuda.stream(streams[1]):
            got[1].append(pg.kvs_paged_extend(qe, *args, pos, cu))
    torch.cuda.synchronize()
    for a, b in zip(*got):
        for x, y in zip((*a, *b), want):
            assert torch.equal(x, y)


def test_long_rows_among_many_short_ones(pg):
    """11 blocks of 128 rows over 262,144 places, which the plan wants to cut into many units, beside 200 jobs of 16 rows,
    for which row blocks are counted that there are not: what is cut has room for its partial results.  The long table
    names 64 blocks 64 times, so that softmax gives what it gives over one time, and LSE ln 64 more."""
    H, D, bs, nb, times, n, S = 64, 64, 64, 64, 64, 1400, 201
    g = torch.Generator().manual_seed(11)
    k, v = (torch.randn(nb, H, bs, D, generator=g).bfloat16() for _ in range(2))
    q = torch.randn(n + 16 * (S - 1), H, D, generator=g).bfloat16()
    table = torch.zeros(S, nb * times, dtype=torch.int32)
    table[0] = torch.arange(nb).repeat(times)
    table[1:, 0] = torch.arange(S - 1) % nb
    blocks = torch.ones(S, dtype=torch.int32)
    blocks[0] = nb * times
    pos = torch.arange(nb * bs, dtype=torch.int32)
    at = torch.cat([torch.arange(n) + nb * bs - n] + [bs * (i % nb) + bs - 16 + torch.arange(16) for i in range(S - 1)]).int()
    cu = torch.cat([torch.zeros(1), n + 16 * torch.arange(S)]).int()
    dev = lambda *x: [t.to(DEV) for t in x]
    o, lse = torch.full_like(q, float("nan")).to(DEV), torch.full(q.shape[:2], float("nan"), device=DEV)
    pg.kvs_paged_extend(*dev(q, k, v, pos, table, blocks, at, cu), out=o, lse=lse)
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    o, lse = o.cpu(), lse.cpu()
    rows = lambda x, b: x[b].transpose(-3, -2).reshape(-1, H, D)
    for h in (0, 31, 63):
        one = slice(h, h + 1)
        want = ref.attend(q[:n, one], rows(k, slice(None))[:, one], rows(v, slice(None))[:, one], D ** -0.5,
                          torch.arange(nb * bs)[None] <= at[:n, None])
        # 64 times as many entries: their sums' share of the bounds, with E <= max |v|
        more = 2 * nb * bs * times * ref.U
        want = (want[0], want[1] + math.log(times), want[2] + more * v.float().abs().max().item(), want[3] + more)
        ref.check(f"long, head {h}", o[:n, one], lse[:n, one], want)
        for i in (0, 63, 199):
            r0 = n + 16 * i
            kb, vb = (rows(x, slice(i % nb, i % nb + 1))[:, one] for x in (k, v))
            see = torch.arange(bs)[None] + bs * (i % nb) <= at[r0:r0 + 16, None]
            ref.check(f"short {i}, head {h}", o[r0:r0 + 16, one], lse[r0:r0 + 16, one],
                      ref.attend(q[r0:r0 + 16, one], kb, vb, D ** -0.5, see))


@pytest.mark.parametrize("n,D", [(1, 128), (1, 64), (40, 128), (40, 64)])
def test_a_position_behind_all_others(pg, n, D):
    """q_pos INT32_MAX sees every entry, and nothing else: 70 entries leave part of a tile empty, whatever its rows."""
    r = Rollouts(pg, 1, 8, 16, 8, 2, D, 5)
    r.append(0, range(70))
    q = r.randn(n, 8, D)
    at = [2 ** 31 - 1] * n
    o, lse = r.cache.extend(q.to(DEV), at, [n])
    r.check_extend(f"INT32_MAX n={n} D={D}", q, o, lse, D ** -0.5, [n], at)
