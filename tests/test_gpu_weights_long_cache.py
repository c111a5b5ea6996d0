"""Weights of entries behind the 2^25 slots that the plan of the decode tells apart (MI355X)."""
import math

import numpy as np
import pytest
import torch

from paper_2609_35750_amd import inputs
from tests import operators_ref as ref
from tests.gpu_helpers import announce, assert_close, assert_lse, to_f64
from tests.test_gpu_weights import DEV, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [0, 1 << 29], ids=["all", "window"])
def test_entries_behind_2_25_slots_get_their_weight(window):
    """A sequence of 2^25 + 640 slots, most of them dead, and one behind it: weights of both, against 64 bits."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import paged as pg

    announce(f"weights behind 2^25 slots, window {window}")
    Hq, Hkv, D, block = 4, 1, 64, 64
    n0, n1 = (1 << 25) // block + 10, 4
    nb = n0 + n1
    rng = np.random.default_rng(1)
    edge = 1 << 25
    live = [np.concatenate([rng.choice(900, 60, replace=False), rng.choice(edge - 2000, 40, replace=False) + 1000,
                            edge - 32 + np.arange(64), edge + 32 + rng.choice(600, 80, replace=False)]),
            n0 * block + rng.choice(n1 * block, 200, replace=False)]
    live = [np.unique(x) for x in live]
    at = torch.from_numpy(np.concatenate(live)).to(DEV)
    k, v = inputs.randn_bf16((len(at), Hkv, D), 1), inputs.randn_bf16((len(at), Hkv, D), 2)
    kc, vc = (torch.zeros((nb, Hkv, block, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    kc.view(nb * block, D)[at], vc.view(nb * block, D)[at] = k.to(DEV)[:, 0], v.to(DEV)[:, 0]
    slot_pos = torch.full((nb * block,), -1, dtype=torch.int32, device=DEV)
    slot_pos[at] = torch.arange(len(at), dtype=torch.int32, device=DEV)
    weight = torch.full((nb * block,), 0.5, device=DEV)
    table = torch.zeros((2, n0), dtype=torch.int32, device=DEV)
    table[0] = torch.arange(n0, dtype=torch.int32, device=DEV)
    table[1, :n1] = torch.arange(n0, nb, dtype=torch.int32, device=DEV)
    nblk = torch.tensor([n0, n1], dtype=torch.int32, device=DEV)
    q = inputs.randn_bf16((2, Hq, D), 3)
    kw = dict(window=window, q_pos=torch.full((2,), len(at), dtype=torch.int32, device=DEV)) if window else {}
    o, lse = pg.kvs_paged_decode_ex(q.to(DEV), kc, vc, slot_pos, table, nblk, slot_weight=weight, **kw)
    torch.cuda.synchronize()
    got = to_f64(weight[at])
    touched = int((weight != 0.5).sum())
    first = 0
    for s, x in enumerate(live):
        mine = slice(first, first + len(x))
        first += len(x)
        one = lambda t: ref.f64(t[mine])[:, :, None, :]  # noqa: E731  (blocks of one slot)
        ro, rl, w, err = ref.decode(ref.f64(q[s]), one(k), one(v), list(range(len(x))), 1, 1.0 / math.sqrt(D))
        assert_close(f"O seq {s}", to_f64(o[s]), ro)
        assert_lse(f"seq {s}", to_f64(lse[s]), rl)
        _within(f"seq {s}", got[mine], 0.5 + w, err + ref.U32 * (0.5 + w))
    assert touched == len(at)
