"""kap_shared_prefix_attn with a q_indptr that is not the schedule's: reported, and the rows behind it are left alone.  All arrays
have the scheduled rows here."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap
from test_gpu_shared_prefix import Case, PAGE

pytestmark = pytest.mark.gpu


def call(c, q_indptr, lse=True):
    q, _, pool, bti, btp, ctx = c.arrays()
    out, sums = torch.full_like(q, 3.0), torch.full(q.shape[:2], 5.0, device=gu.DEV)
    kap.shared_prefix_attn(q, gu.i32(q_indptr), pool, bti, btp, ctx, out, c.ws, lse=sums if lse else None)
    with pytest.raises(kap.KapError) as e:
        c.ws.check()
    assert e.value.code == kap.ERR_DEVICE_INDEX
    return out, sums


GROUPS = [[(3, [(4, 20), (4, 9)])], [(30, [(4, 20 + i) for i in range(40)])], [(21, [(4, 9)] * 70), (0, [(4, 50)] * 3)]]


@pytest.mark.parametrize("hq,hkv", [(8, 2), (2, 2), (16, 1)])
@pytest.mark.parametrize("groups", GROUPS)
def test_fewer_rows_than_scheduled(groups, hq, hkv):
    c = Case(50, groups, hq, hkv, poison=0.0)
    c.ws = c.workspace()
    batch = len(c.n_q)
    for n_q in (np.full(batch, 1), np.full(batch, 3), np.concatenate([np.full(batch - 1, 4), [3]])):
        indptr = np.concatenate([[0], np.cumsum(n_q)])
        out, lse = call(c, indptr)
        end = int(indptr[-1])
        assert (out[end:] == 3.0).all() and (lse[end:] == 5.0).all()
        out, _ = call(c, indptr, lse=False)
        assert (out[end:] == 3.0).all()
    call(c, np.zeros(batch + 1))
    assert (call(c, np.zeros(batch + 1))[0] == 3.0).all()
    c.check()                                                                    # the schedule's own rows, after all that


def test_more_rows_than_scheduled_are_reported():
    c = Case(51, GROUPS[1], poison=0.0)
    c.ws = c.workspace()
    indptr = c.q_indptr.copy()
    indptr[-1] += 2
    call(c, indptr)
    c.check()


@pytest.mark.parametrize("place", ["q_indptr", "bt_indptr", "bt_pages", "ctx_len", "lse", "q", "out", "pool"])
def test_misaligned_arrays_are_refused(place):
    c = Case(52, GROUPS[0], poison=0.0)
    c.ws = c.workspace()
    q, qi, pool, bti, btp, ctx = c.arrays()
    out, lse = torch.full_like(q, 3.0), torch.zeros(q.shape[:2], device=gu.DEV)
    at = dict(q=q.data_ptr(), q_indptr=qi.data_ptr(), pool=pool.data_ptr(), bt_indptr=bti.data_ptr(), bt_pages=btp.data_ptr(), ctx_len=ctx.data_ptr(),
              out=out.data_ptr(), lse=lse.data_ptr())
    at[place] += 2
    code = kap.lib().kap_shared_prefix_attn(at["q"], at["q_indptr"], at["pool"], pool.shape[0], at["bt_indptr"], at["bt_pages"], at["ctx_len"], 2, c.hq, c.hkv,
                                            128, PAGE, c.scale, at["out"], at["lse"], c.ws._h, torch.cuda.current_stream().cuda_stream)
    assert code == kap.ERR_INVALID_ARG and b"aligned" in kap.lib().kap_last_error()
    torch.cuda.synchronize()
    assert (out == 3.0).all()
