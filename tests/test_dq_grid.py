"""The dQ kernel's grid where its row workgroups leave no room in a launch for those that add up split key blocks: as plain
arithmetic on the CPU, and on the GPU (MI355X) through short traces under a bound on their length of nearly a million."""
import shutil

import numpy as np
import pytest
import torch

from tests.test_device_host import HIPCC, _build_and_run

DEV = "cuda:0"


@pytest.mark.skipif(HIPCC is None or shutil.which("g++") is None, reason="hipcc not available")
def test_sums_ride_along_exactly_where_they_fit(tmp_path):
    r = _build_and_run(tmp_path, "dq_grid.hip", "dq_grid")
    assert r.returncode == 0 and r.stdout.rstrip().endswith("ok"), r.stdout + r.stderr


@pytest.mark.gpu
@pytest.mark.parametrize("window", [0, 5000], ids=["evict", "window"])
def test_backward_under_a_launch_full_of_row_workgroups(window):
    """256 traces, one of them long enough to have split key blocks: 2^24 - 512 row workgroups under max_seqlen 2^20 - 32,
    and the same traces under their true bound.  The two differ in the grid alone."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import kvs
    from tests.gpu_helpers import announce

    announce(f"backward, 2^24 - 512 row workgroups, window {window}")
    rng = np.random.default_rng(0)
    lengths = np.concatenate([[9000], rng.integers(0, 30, 255)])
    cu = torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)).to(DEV)
    n, Hq, Hkv, D = int(lengths.sum()), 8, 2, 64
    gen = torch.Generator(device=DEV).manual_seed(1)
    q, do = (torch.randn(n, Hq, D, generator=gen, device=DEV).bfloat16() for _ in range(2))
    k, v = (torch.randn(n, Hkv, D, generator=gen, device=DEV).bfloat16() for _ in range(2))
    e = torch.full((n,), 2 ** 31 - 1, dtype=torch.int32, device=DEV)
    out = []
    for mx in (9000, (1 << 20) - 32):
        kw = dict(cu_seqlens=cu, max_seqlen=mx)
        if window:
            o, lse = kvs.kvs_window_attn_fwd(q, k, v, window, 4, e, **kw)
            g = kvs.kvs_window_attn_bwd(do, q, k, v, o, lse, window, 4, e, **kw)
        else:
            o, lse = kvs.kvs_evict_attn_fwd(q, k, v, e, **kw)
            g = kvs.kvs_evict_attn_bwd(do, q, k, v, o, lse, e, **kw)
        torch.cuda.synchronize()
        out.append([o, lse, *g])
    for name, a, b in zip(("O", "LSE", "dQ", "dK", "dV"), *out):
        assert torch.equal(a, b), name
