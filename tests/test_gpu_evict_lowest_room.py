"""Eviction of the lowest with room for as many positions as a 32-bit count can say (MI355X)."""
import numpy as np
import pytest
import torch

from tests import operators_ref as ref
from tests.gpu_helpers import announce
from tests.test_gpu_weights import DEV, _cache, _dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("keep", [60, 10 ** 6], ids=["some leave", "none leaves"])
def test_the_rest_of_the_longest_list_is_filled(keep):
    """2^31 - 1 places for one sequence's positions: those that left, then -1 up to the last."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import paged as pg

    announce(f"evict lowest: room for 2^31 - 1, keep {keep}")
    c = _cache(1, 300, 300, 16, 1, 64, 2)
    d = _dev(c)
    pos, counts = pg.kvs_paged_evict_lowest(d["weight"], d["slot_pos"], d["table"], d["nblk"],
                                            torch.tensor([keep], dtype=torch.int32, device=DEV), 16, max_out=2 ** 31 - 1)
    torch.cuda.synchronize()
    gone = ref.evict_lowest(c["weight"].numpy(), c["slot_pos"], c["table"][0], c["nblk"][0], 16, c["nb"], keep, 0, 0, 10 ** 6)
    assert int(counts[0]) == len(gone)
    np.testing.assert_array_equal(pos[0, :len(gone)].cpu().numpy(), c["slot_pos"][gone])
    assert all(bool((part == -1).all()) for part in pos[0, len(gone):].split(1 << 28))
