"""Row workgroups beyond what a launch holds are refused, not counted modulo 2^32 (MI355X)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_more_row_workgroups_than_a_launch_holds_are_refused():
    """2,049 traces of one token under max_seqlen 2^20 with 64 KV heads: 2^32 + 2^21 row workgroups."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_35750_amd import kvs
    from tests.gpu_helpers import announce

    announce("2^32 + 2^21 row workgroups")
    B, Hq, Hkv, D = 2049, 256, 64, 64
    cu = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    q = torch.ones(B, Hq, D, device=DEV).bfloat16()
    k = torch.ones(B, Hkv, D, device=DEV).bfloat16()
    e = torch.full((B,), 2 ** 31 - 1, dtype=torch.int32, device=DEV)
    lse = torch.zeros(Hq, B, device=DEV)
    kw = dict(cu_seqlens=cu, max_seqlen=1 << 20)
    for call in (lambda: kvs.kvs_evict_attn_fwd(q, k, k, e, **kw), lambda: kvs.kvs_window_attn_fwd(q, k, k, 8, 0, e, **kw),
                 lambda: kvs.kvs_evict_attn_bwd(q, q, k, k, q, lse, e, **kw),
                 lambda: kvs.kvs_window_attn_bwd(q, q, k, k, q, lse, 8, 0, e, **kw)):
        with pytest.raises(kvs.KvsError) as err:
            call()
        assert err.value.status == kvs.KVS_ERR_HIP
    torch.cuda.synchronize()
    o, _ = kvs.kvs_evict_attn_fwd(q, k, k, e, cu_seqlens=cu, max_seqlen=1)     # the next call is not touched by them
    torch.cuda.synchronize()
    np.testing.assert_array_equal(o.float().cpu().numpy(), np.ones((B, Hq, D), dtype=np.float32))
