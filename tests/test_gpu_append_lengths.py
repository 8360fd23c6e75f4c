"""kap_append_kv with a negative ctx_len: reported, and neither its block table in front of the first entry nor anything else is touched."""
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("length", [-1, -16, -1000, -2 ** 31])
@pytest.mark.parametrize("n_new", [1, 20])
def test_a_negative_length_is_reported(length, n_new):
    hkv, pages, status = 2, 12, torch.zeros(1, dtype=torch.int32, device=gu.DEV)
    k, v = (torch.randn((n_new + 1, hkv, 128), device=gu.DEV).to(torch.bfloat16) for _ in range(2))
    pool = torch.full((pages, 2, hkv, 16, 128), 3.0, dtype=torch.bfloat16, device=gu.DEV)
    kap.append_kv(k, v, pool, gu.i32([0, 2, 4]), gu.i32([5, 6, 7, 8]), gu.i32([length, 3]), new_indptr=gu.i32([0, n_new, n_new + 1]), advance=False, device_status=status)
    assert int(status[0]) == 1 << kap.ERR_DEVICE_INDEX
    assert torch.equal(pool[7, 0, :, 3], k[n_new]) and torch.equal(pool[7, 1, :, 3], v[n_new])
    pool[7, :, :, 3] = 3.0
    assert bool((pool == 3.0).all())
