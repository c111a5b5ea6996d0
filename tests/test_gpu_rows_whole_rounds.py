"""New tokens whose row blocks fill more than a round of the chip (MI355X): those of whole rounds are left whole and write
their rows, the ones behind them are cut and joined, and where one kind ends and the other begins lies inside a token's
q-heads where 128 is no multiple of their number."""
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


# New tokens and entries a sequence; places on the chip: 768 / Hkv a KV head, so 12 row blocks of 128 rows fill a round at
# Hkv = 64 and 24 at Hkv = 32.  Row blocks left whole, and the units of those that are cut, without a window: 12 and 2 x 2;
# 12 and 5 x 2; 12 and 3 x 4; 24 and 5 x 3; 24 and 4 x 4; 24 and 8 x 2; 24 and 4 x 4; 12 and 5 x 2 (more sequences than one
# wave plans).  Under the window the first, fifth, seventh and last are cut so too, the others into one unit a row block.
CASES = [
    ([1700], [1700], 64, 64, 64),
    ([900, 1100], [1500, 1900], 64, 64, 64),
    ([1000, 801], [3000, 2500], 64, 64, 128),
    ([600, 575], [2000, 1500], 96, 32, 128),
    ([700, 3], [2500, 900], 160, 32, 64),
    ([333, 444], [1333, 2444], 160, 32, 64),
    ([700], [3000], 160, 32, 128),
    ([1] * 270 + [1500, 600], [20] * 270 + [1700, 2600], 64, 64, 64),
]


@pytest.mark.parametrize("window,sinks", [(None, 0), (200, 5)])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{max(c[0])}_H{c[2]}x{c[3]}_D{c[4]}")
def test_row_blocks_beyond_a_round(pg, case, window, sinks):
    announce(f"row blocks beyond a round, {max(case[0])} of {len(case[0])}, {case[2:]}, window {window}")
    new, ends, Hq, Hkv, D = case
    S, bs, G = len(new), 16, Hq // Hkv
    n = sum(new)
    g = torch.Generator().manual_seed(Hq + D + n)
    count = [-(-e // bs) for e in ends]
    order = torch.randperm(sum(count) + 2, generator=g).int()
    table, pos = torch.zeros(S, max(count), dtype=torch.int32), torch.full((len(order), bs), -1, dtype=torch.int32)
    at = 0
    for s, (e, c) in enumerate(zip(ends, count)):
        table[s, :c] = order[at:at + c]
        mine = torch.arange(c * bs, dtype=torch.int32).view(c, bs)
        mine[mine >= e] = -1
        mine[(mine % 37 == 5) & (mine < e - new[s])] = -1          # evicted ones
        pos[order[at:at + c].long()] = mine
        at += c
    k, v = (torch.randn(len(order), Hkv, bs, D, generator=g).bfloat16() for _ in range(2))
    dead = (pos < 0)[:, None, :].expand(-1, Hkv, -1)
    k[dead], v[dead] = float("nan"), float("inf")
    q = torch.randn(n, Hq, D, generator=g).bfloat16()
    q_pos = torch.cat([torch.arange(e - x, e) for e, x in zip(ends, new)]).int()
    cu = torch.tensor([0] + new).cumsum(0).int()
    o, lse = torch.full_like(q, float("nan")).to(DEV), torch.full((n, Hq), float("nan"), device=DEV)
    pg.kvs_paged_extend(*(t.to(DEV) for t in (q, k, v, pos.view(-1), table, torch.tensor(count).int(), q_pos, cu)),
                        window=window, sinks=sinks, out=o, lse=lse)
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    o, lse = o.cpu(), lse.cpu()
    heads = sorted(set(range(G, 2 * G)) | {0, Hq - 1})               # all of one KV head, and two others
    for s in sorted({0, S // 2, S - 2, S - 1} & set(range(S))):
        blocks = table[s, :count[s]].long()
        live = (pos[blocks] >= 0).view(-1)
        p, i = pos[blocks].view(-1)[live][None], q_pos[cu[s]:cu[s + 1], None]
        see = p <= i
        if window:
            see &= (i - p < window) | (p < sinks)
        rows = slice(int(cu[s]), int(cu[s + 1]))
        for h in heads:
            kv = [x[blocks, h // G].reshape(-1, 1, D)[live] for x in (k, v)]
            one = slice(h, h + 1)
            ref.check(f"seq {s} head {h}", o[rows, one], lse[rows, one], ref.attend(q[rows, one], *kv, D ** -0.5, see))
