"""Sequences that share cache blocks, CPU tier: the block manager's forks,
copies, evictions in shared blocks, compactions and groups against a plain model
of what every sequence holds, on a simulated device; refusals of the calls.
"""
import ctypes
import itertools
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_35750_amd", "libkvs.so")

pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="libkvs.so not built (run __graft_entry__.build())")


@pytest.fixture(scope="module")
def paged():
    from paper_2609_35750_amd import paged as p

    return p


class Device:
    """Slots as the device holds them: position (-1: none) and content."""

    def __init__(self, bm):
        self.bm, n = bm, bm.num_blocks * bm.block_size
        self.pos, self.content = np.full(n, -1), np.full(n, -1)

    def append(self, seq, positions, contents):
        slots = self.bm.append(seq, positions)
        assert (self.pos[slots] == -1).all(), "an append's slots hold no entry"
        self.pos[slots], self.content[slots] = positions, contents

    def evict(self, seq, positions):
        slots, (src, dst) = self.bm.evict_shared(seq, positions)
        self.pos[slots[slots >= 0]] = -1
        self.copy(src, dst)
        return len(src)

    def copy(self, src, dst, move=False):
        assert len(set(dst)) == len(dst) and not set(src) & set(dst)
        assert (self.pos[src] >= 0).all() and (self.pos[dst] == -1).all()
        self.pos[dst], self.content[dst] = self.pos[src], self.content[src]
        if move:
            self.pos[src] = -1

    def release(self, seq):
        self.pos[self.bm.release(seq)] = -1

    def holds(self, seq):
        table, n = self.bm.tables()
        bs = self.bm.block_size
        slots = (table[seq, :n[seq], None] * bs + np.arange(bs)).reshape(-1)
        slots = slots[self.pos[slots] >= 0]
        assert len(set(self.pos[slots])) == len(slots)
        return dict(zip(self.pos[slots].tolist(), self.content[slots].tolist()))


def check(dev, model):
    bm = dev.bm
    table, n = bm.tables()
    for s, want in enumerate(model):
        assert dev.holds(s) == want
        assert bm.live(s) == len(want)
    used = {b for s in range(len(model)) for b in table[s, :n[s]].tolist()}
    assert bm.free_blocks() == bm.num_blocks - len(used)
    for s in range(len(model)):
        others = {b for t in range(len(model)) if t != s for b in table[t, :n[t]].tolist()}
        assert bm.shared(s) == sum(b in others for b in table[s, :n[s]].tolist())
    # nothing is live outside the tables
    bs = bm.block_size
    live = set((np.flatnonzero(dev.pos >= 0) // bs).tolist())
    assert live <= used


@pytest.mark.parametrize("bs", [1, 2, 5, 16, 64])
@pytest.mark.parametrize("seed", range(6))
def test_random_histories(paged, bs, seed):
    rng = np.random.default_rng([seed, bs])
    S = 5
    dev = Device(paged.BlockManager(4000 // bs + 20, bs, S, 400))
    model = [{} for _ in range(S)]
    nxt = [0] * S
    fresh = itertools.count()
    for _ in range(120):
        s, t = (int(x) for x in rng.choice(S, 2, replace=False))
        op = rng.choice(["append", "append", "evict", "evict", "span", "fork", "fork", "copy", "compact", "release"])
        if op == "append":
            n = int(rng.integers(0, 40))
            p = nxt[s] + np.arange(n)
            c = [next(fresh) for _ in range(n)]
            dev.append(s, p, c)
            model[s].update(zip(p.tolist(), c))
            nxt[s] += n
        elif op in ("evict", "span") and model[s]:
            have = sorted(model[s])
            if op == "evict":
                gone = rng.choice(have, int(rng.integers(0, min(len(have), 30) + 1)), replace=False)
            else:
                a, b = sorted(rng.integers(0, len(have) + 1, 2))
                gone = rng.permutation(have[a:b])
            dev.evict(s, gone.astype(np.int32))
            for p in gone.tolist():
                del model[s][p]
        elif op in ("fork", "copy"):
            if model[t]:
                dev.release(t)
                model[t] = {}
            if op == "fork":
                dev.bm.fork(s, t)
            else:
                dev.copy(*dev.bm.copy(s, t))
            model[t], nxt[t] = dict(model[s]), nxt[s]
        elif op == "compact":
            tab, n = dev.bm.tables()
            dev.copy(*dev.bm.compact(s), move=True)
            # as few blocks as hold what is the sequence's own, but for one with room for appends
            tab, n = dev.bm.tables()
            own = len(tab[s, :n[s]]) - dev.bm.shared(s)
            shared = sum(int((dev.pos.reshape(-1, bs)[b] >= 0).sum()) for b in tab[s, :n[s]].tolist()
                         if any(b in tab[o, :n[o]].tolist() for o in range(S) if o != s))
            assert own <= -(-(len(model[s]) - shared) // bs) + 1
        elif op == "release":
            dev.release(s)
            model[s], nxt[s] = {}, int(rng.integers(0, 10))
        check(dev, model)
    for s in range(S):
        dev.release(s)
    assert dev.bm.free_blocks() == dev.bm.num_blocks and (dev.pos == -1).all()


def test_fork_copies_nothing_and_seals_the_last_block(paged):
    dev = Device(paged.BlockManager(20, 4, 2, 10))
    dev.append(0, range(6), range(6))
    free = dev.bm.free_blocks()
    dev.bm.fork(0, 1)
    assert dev.bm.free_blocks() == free and dev.bm.shared(0) == dev.bm.shared(1) == 2
    table, n = dev.bm.tables()
    np.testing.assert_array_equal(table[0, :2], table[1, :2])
    dev.append(0, [6], [60])
    dev.append(1, [6], [61])
    check(dev, [dict(zip(range(7), [0, 1, 2, 3, 4, 5, 60])), dict(zip(range(7), [0, 1, 2, 3, 4, 5, 61]))])
    assert dev.bm.shared(0) == 2


def test_span_of_whole_shared_blocks_needs_no_copy(paged):
    dev = Device(paged.BlockManager(20, 4, 2, 10))
    dev.append(0, range(16), range(16))
    dev.bm.fork(0, 1)
    assert dev.evict(1, np.arange(4, 12)) == 0
    check(dev, [{p: p for p in range(16)}, {p: p for p in (0, 1, 2, 3, 12, 13, 14, 15)}])
    assert dev.evict(1, np.array([0])) == 3
    check(dev, [{p: p for p in range(16)}, {p: p for p in (1, 2, 3, 12, 13, 14, 15)}])
    # the other sequence's blocks are its own again where nobody else holds them
    assert dev.bm.shared(0) == 1
    assert dev.evict(0, np.array([0, 5])) == 0


def test_old_evict_refuses_what_needs_copies(paged):
    from paper_2609_35750_amd.kvs import KVS_ERR_STATE, KvsError

    dev = Device(paged.BlockManager(20, 4, 2, 10))
    dev.append(0, range(8), range(8))
    dev.bm.fork(0, 1)
    with pytest.raises(KvsError) as e:
        dev.bm.evict(1, [0, 1, 2])
    assert e.value.status == KVS_ERR_STATE
    check(dev, [{p: p for p in range(8)}] * 2)
    np.testing.assert_array_equal(dev.bm.evict(1, [0, 1, 2, 3]), [-1] * 4)
    check(dev, [{p: p for p in range(8)}, {p: p for p in range(4, 8)}])


def test_refusals_leave_the_manager_as_it_was(paged):
    from paper_2609_35750_amd.kvs import KVS_ERR_CAPACITY, KVS_ERR_SHAPE, KVS_ERR_STATE, KvsError

    def refused(status, call, *args):
        with pytest.raises(KvsError) as e:
            call(*args)
        assert e.value.status == status
        check(dev, model)

    dev = Device(paged.BlockManager(5, 4, 3, 4))
    dev.append(0, range(10), range(10))
    dev.append(1, range(3), range(3))
    model = [{p: p for p in range(10)}, {p: p for p in range(3)}, {}]
    bm = dev.bm
    for call in (bm.fork, bm.copy):
        refused(KVS_ERR_SHAPE, call, 0, 0)
        refused(KVS_ERR_SHAPE, call, 0, 3)
        refused(KVS_ERR_SHAPE, call, -1, 2)
        refused(KVS_ERR_STATE, call, 0, 1)
    refused(KVS_ERR_CAPACITY, bm.copy, 0, 2)
    refused(KVS_ERR_SHAPE, bm.compact, 3)
    bm.fork(0, 2)
    model[2] = dict(model[0])
    refused(KVS_ERR_CAPACITY, bm.evict_shared, 2, [0, 5])          # two blocks to replace, one is free
    refused(KVS_ERR_STATE, bm.evict_shared, 2, [0, 0])
    refused(KVS_ERR_STATE, bm.evict_shared, 2, [0, 77])
    refused(KVS_ERR_STATE, bm.evict_shared, 2, [-1])
    assert dev.evict(2, np.array([0])) == 3
    del model[2][0]
    check(dev, model)
    assert bm.shared(5) == bm.shared(-1) == -1


def _saving(bm, group, blocks):
    return sum((int((group == g).sum()) - 1) * int(b) for g, b in enumerate(blocks))


def _best(lists):
    """Most block reads saved where all tables that begin alike are one group, or fall into groups by how they go on."""
    common = len(os.path.commonprefix(lists)) if len(lists) > 1 else 0
    inside = {}
    for x in lists:
        if len(x) > common:
            inside.setdefault(x[common], []).append(x)
    return max((len(lists) - 1) * common, sum(_best(x) for x in inside.values() if len(x) > 1))


@pytest.mark.parametrize("seed", range(25))
def test_groups_save_most(paged, seed):
    rng = np.random.default_rng(seed)
    S = 6
    bm = paged.BlockManager(400, 2, S, 60)
    at = [0] * S

    def grow(s):
        n = int(rng.integers(0, 12))
        bm.append(s, at[s] + np.arange(n))
        at[s] += n

    grow(0)
    for s in range(1, S):
        if rng.random() < 0.8:
            src = int(rng.integers(0, s))
            bm.fork(src, s)
            at[s] = at[src]
            grow(src)
        grow(s)
    if rng.random() < 0.5:
        s = int(rng.integers(0, S))
        if at[s]:
            bm.evict_shared(s, [int(rng.integers(0, at[s]))])
    group, blocks = bm.groups()
    table, n = bm.tables()
    assert set(group.tolist()) <= set(range(-1, len(blocks))) and (blocks > 0).all()
    lists = [table[s, :n[s]].tolist() for s in range(S)]
    for g, b in enumerate(blocks):
        members = [lists[s] for s in range(S) if group[s] == g]
        assert len(members) > 1 and all(m[:b] == members[0][:b] and len(m) >= b for m in members)
    assert _saving(bm, group, blocks) == _best(lists)


def test_groups_of_nothing_shared(paged):
    bm = paged.BlockManager(10, 4, 3, 5)
    bm.append(0, range(5))
    group, blocks = bm.groups()
    assert (group == -1).all() and blocks.size == 0


def test_null_arguments(paged):
    from paper_2609_35750_amd.kvs import KVS_ERR_NULL, KVS_ERR_SHAPE, lib

    bm = paged.BlockManager(10, 4, 3, 5)
    bm.append(0, range(5))
    n = ctypes.c_int()
    buf = np.zeros(16, dtype=np.int32).ctypes.data
    assert lib.kvs_bm_fork(None, 0, 1) == KVS_ERR_NULL
    assert lib.kvs_bm_copy(bm._h, 0, 1, None, buf, ctypes.byref(n)) == KVS_ERR_NULL
    assert lib.kvs_bm_copy(bm._h, 0, 1, buf, buf, None) == KVS_ERR_NULL
    assert lib.kvs_bm_compact(bm._h, 0, None, None, ctypes.byref(n)) == KVS_ERR_NULL
    assert lib.kvs_bm_evict_shared(bm._h, 0, buf, 1, buf, None, buf, ctypes.byref(n)) == KVS_ERR_NULL
    assert lib.kvs_bm_evict_shared(bm._h, 0, buf, -1, buf, buf, buf, ctypes.byref(n)) == KVS_ERR_SHAPE
    assert lib.kvs_bm_groups(bm._h, buf, None, ctypes.byref(n)) == KVS_ERR_NULL
    assert lib.kvs_bm_shared(None, 0) == -1


FAKE = 1 << 20   # 16-byte aligned, never dereferenced: validation fails first


def _shared(lib, S=4, groups=1, Hq=8, Hkv=2, D=64, nb=10, bs=16, mb=4, q=FAKE, group=FAKE, blocks=FAKE, ws=FAKE,
            ws_bytes=1 << 40, scale=0.125):
    return lib.kvs_paged_decode_shared(q, FAKE, FAKE, FAKE, FAKE, FAKE, group, blocks, FAKE, FAKE, S, groups, Hq, Hkv, D, nb,
                                       bs, mb, scale, ws, ws_bytes, None)


def _extend(lib, S=4, n=16, Hq=8, Hkv=2, D=64, nb=10, bs=16, mb=4, q=FAKE, pos=FAKE, cu=FAKE, ws=FAKE, ws_bytes=1 << 40,
            scale=0.125, window=0, sinks=0):
    return lib.kvs_paged_extend(q, FAKE, FAKE, FAKE, FAKE, FAKE, pos, cu, FAKE, FAKE, S, n, Hq, Hkv, D, nb, bs, mb, scale,
                                window, sinks, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_shared, _extend])
def test_attention_refusals(paged, call):
    from paper_2609_35750_amd import kvs as k

    lib = k.lib
    for bad in ({"Hq": 6, "Hkv": 4}, {"D": 96}, {"S": 0}, {"Hkv": 0}, {"bs": 65}, {"bs": 0}, {"nb": 0}, {"mb": 0},
                {"scale": 0.0}, {"scale": float("inf")}, {"scale": float("nan")}, {"scale": -1.0}):
        assert call(lib, **bad) == k.KVS_ERR_SHAPE, bad
    for bad in ({"Hq": 130, "Hkv": 2}, {"nb": 1 << 30, "bs": 1, "Hkv": 8}, {"mb": 1 << 27, "bs": 16}, {"S": 1 << 26, "n": 1 << 26}
                if call is _extend else {"S": 1 << 26}):
        assert call(lib, **bad) == k.KVS_ERR_UNSUPPORTED, bad
    assert call(lib, q=None) == k.KVS_ERR_NULL
    assert call(lib, q=FAKE + 8) == k.KVS_ERR_ALIGN
    assert call(lib, ws=FAKE + 8) == k.KVS_ERR_ALIGN
    assert call(lib, ws_bytes=100) == k.KVS_ERR_WORKSPACE
    assert call(lib, ws=None) == k.KVS_ERR_NULL


def test_refusals_of_each(paged):
    from paper_2609_35750_amd import kvs as k

    lib = k.lib
    assert _shared(lib, groups=0) == k.KVS_ERR_SHAPE
    assert _shared(lib, group=None) == _shared(lib, blocks=None) == k.KVS_ERR_NULL
    assert _extend(lib, n=-1) == _extend(lib, window=-1) == _extend(lib, sinks=-1) == k.KVS_ERR_SHAPE
    assert _extend(lib, pos=None) == _extend(lib, cu=None) == k.KVS_ERR_NULL
    assert _extend(lib, n=0, q=None, pos=None, cu=None, ws=None, ws_bytes=0) == k.KVS_OK
    for bad in ((0, 1, 1, 64), (1, 0, 1, 64), (1, 1, 0, 64), (1, 1, 1, 0)):
        assert lib.kvs_paged_decode_shared_workspace(bad[0], 1, bad[1], bad[2], bad[3], 4, 16) == 0
        assert lib.kvs_paged_extend_workspace(bad[0], 5, bad[1], bad[2], bad[3], 4, 16) == 0

    def copy(src=FAKE, dst=FAKE, n=3, kc=FAKE, pos=FAKE, move=0, nb=10, bs=16, Hkv=2, D=64):
        return lib.kvs_paged_copy(src, dst, n, kc, FAKE, pos, None, move, nb, bs, Hkv, D, None)

    assert copy(n=-1) == copy(Hkv=0) == copy(D=32) == copy(bs=65) == copy(nb=0) == k.KVS_ERR_SHAPE
    assert copy(src=None) == copy(dst=None) == copy(kc=None) == copy(pos=None, move=1) == k.KVS_ERR_NULL
    assert copy(kc=FAKE + 4) == k.KVS_ERR_ALIGN
    assert copy(nb=1 << 30, bs=4) == k.KVS_ERR_UNSUPPORTED
    assert copy(n=0, src=None, dst=None) == k.KVS_OK


def test_out_of_memory(tmp_path):
    """Host only: a failed allocation in a fork, a copy, a shared eviction, a compaction or the groups gives an error and
    leaves the manager as it was."""
    src = os.path.join(ROOT, "paper_2609_35750_amd", "csrc")
    exe = str(tmp_path / "bm_share_memory")
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", src, os.path.join(ROOT, "tests", "host", "bm_share_memory.cpp"),
                    os.path.join(src, "kvs_cache.cpp"), "-o", exe], check=True, capture_output=True, text=True)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.endswith("ok\n"), out.stdout
