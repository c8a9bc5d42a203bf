"""The 8-bit paged cache at its edges: waits that run out, instances and calls that the other tests pass by."""
import numpy as np
import pytest
import torch

from paper_2609_34606_b200 import hsa
from test_kv8 import Case, dev_i32


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,counts,lengths", [(2, 2, [1], [20000]), (4, 2, [2, 7], [300, 9000]), (16, 1, [1, 1, 0], [5000, 70, 9]),
                                                   (4, 4, [20, 100], [2000, 3001]), (4, 2, [300, 1, 200], [9000, 1, 200]),
                                                   (3, 3, [1] * 200, [700] * 200), (2, 2, [40] * 160, [200] * 160)])
@pytest.mark.parametrize("listed", [False, True])
def test_attention_that_gives_up_leaves_the_context_usable(cuda_device, d, Hq, Hkv, counts, lengths, listed):
    """Waits of the attention kernels run out with copies and products in flight: the kernel ends by itself and says so, and the
    next call gives the usual bits."""
    c = Case(cuda_device, Hq, Hkv, d, lengths, seed=31, max_tokens=sum(lengths))
    c.append(lengths, twin=False)
    sel = None
    if listed:
        sel = [[list(c_) for c_ in [range(h % 2, -(-n // 64), 2)] * Hkv] for h, n in enumerate(lengths)]
    q, want, want_lse = c.attend(counts, True, sel=sel, check=False)
    assert c.cache.device_status() == 0
    for limit in (1, 1, 300, 1000, 3000, 10000, 20_000):
        c.cache.set_wait_limit_ns(limit)
        _, got, lse = c.attend(counts, True, sel=sel, q=q, check=False)
        status = c.cache.device_status()
        assert status == hsa.HSA_ERR_DEVICE_TIMEOUT or limit > 1 and status == 0
        if status == 0:
            assert torch.equal(got, want) and torch.equal(lse, want_lse)
    c.cache.set_wait_limit_ns(2_000_000_000)
    for _ in range(2):
        _, got, lse = c.attend(counts, True, sel=sel, q=q, check=False)
        assert c.cache.device_status() == 0 and torch.equal(got, want) and torch.equal(lse, want_lse)
