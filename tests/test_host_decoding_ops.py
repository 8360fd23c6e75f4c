"""Refusals of kap_append_kv_rope, kap_shared_prefix_items and kap_sample_tokens: argument errors are found on the
host before anything is launched, so they can be seen without a GPU (the pointers are never followed)."""
import ctypes as C

import numpy as np
import pytest

from paper_2607_24260_b200 import kap

A = C.c_void_p(1 << 20)                        # an aligned address that nothing reads
ODD = C.c_void_p((1 << 20) + 2)


def _append(**change):
    a = dict(q=A, qs=4096, k=A, ks=1024, v=A, vs=1024, qo=A, qos=4096, indptr=None, rows=4, freq=A, rot=128, inter=0, pos=None,
             pos_stride=0, axes=0, axis=None, offset=None, pool=A, pages=10, bti=A, btp=A, ctx=A, advance=1, batch=4, hq=32, hkv=8,
             d=128, page=16, layout=0, status=None, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return kap.lib().kap_append_kv_rope(*a.values())


@pytest.mark.parametrize("change,code", [
    (dict(d=64), kap.ERR_UNSUPPORTED), (dict(page=32), kap.ERR_UNSUPPORTED), (dict(rot=0), kap.ERR_UNSUPPORTED),
    (dict(rot=24), kap.ERR_UNSUPPORTED), (dict(rot=144), kap.ERR_UNSUPPORTED), (dict(rot=-16), kap.ERR_UNSUPPORTED),
    (dict(batch=-1), kap.ERR_INVALID_ARG), (dict(rows=-1), kap.ERR_INVALID_ARG), (dict(rows=5), kap.ERR_INVALID_ARG),
    (dict(hkv=0), kap.ERR_INVALID_ARG), (dict(hq=0), kap.ERR_INVALID_ARG), (dict(layout=2), kap.ERR_INVALID_ARG),
    (dict(k=None), kap.ERR_INVALID_ARG), (dict(v=None), kap.ERR_INVALID_ARG), (dict(qo=None), kap.ERR_INVALID_ARG),
    (dict(pool=None), kap.ERR_INVALID_ARG), (dict(pages=0), kap.ERR_INVALID_ARG), (dict(bti=None), kap.ERR_INVALID_ARG),
    (dict(ctx=None), kap.ERR_INVALID_ARG), (dict(freq=None), kap.ERR_INVALID_ARG), (dict(q=ODD), kap.ERR_INVALID_ARG),
    (dict(k=ODD), kap.ERR_INVALID_ARG), (dict(pool=ODD), kap.ERR_INVALID_ARG), (dict(ks=1028), kap.ERR_INVALID_ARG),
    (dict(ks=1016), kap.ERR_INVALID_ARG), (dict(qs=4088), kap.ERR_INVALID_ARG), (dict(qos=0), kap.ERR_INVALID_ARG),
    (dict(axes=2), kap.ERR_INVALID_ARG), (dict(pos=A, axes=0), kap.ERR_INVALID_ARG), (dict(pos=A, axes=3, pos_stride=4), kap.ERR_INVALID_ARG),
    (dict(pos=A, axes=1, pos_stride=4, offset=A), kap.ERR_INVALID_ARG),
])
def test_append_kv_rope_refusals(change, code):
    assert _append(**change) == code
    assert kap.lib().kap_last_error()


def test_append_kv_rope_refuses_an_axis_that_is_not_there():
    axis = (C.c_uint8 * 64)(*([0, 1, 2] * 21 + [3]))
    assert _append(pos=A, axes=3, pos_stride=4, axis=axis) == kap.ERR_INVALID_ARG
    assert b"freq_axis[63] = 3" in kap.lib().kap_last_error()
    assert _append(pos=A, axes=3, pos_stride=3, axis=(C.c_uint8 * 64)()) == kap.ERR_INVALID_ARG     # rows overlap


def test_append_kv_rope_of_nothing():
    assert _append(batch=0, rows=0) == kap.OK
    assert _append(batch=2, rows=0, indptr=A) == kap.OK


def _sample(**change):
    a = dict(logits=A, kind=0, stride=100, rows=2, vocab=100, t=None, k=None, p=None, m=None, u=A, token=A, logprob=None, stream=None)
    assert set(change) <= set(a)
    a.update(change)
    return kap.lib().kap_sample_tokens(*a.values())


@pytest.mark.parametrize("change,code", [
    (dict(kind=2), kap.ERR_UNSUPPORTED), (dict(kind=-1), kap.ERR_UNSUPPORTED), (dict(rows=-1), kap.ERR_INVALID_ARG),
    (dict(vocab=0), kap.ERR_INVALID_ARG), (dict(stride=99), kap.ERR_INVALID_ARG), (dict(logits=None), kap.ERR_INVALID_ARG),
    (dict(u=None), kap.ERR_INVALID_ARG), (dict(token=None), kap.ERR_INVALID_ARG), (dict(logits=ODD), kap.ERR_INVALID_ARG),
    (dict(logits=C.c_void_p((1 << 20) + 1), kind=1), kap.ERR_INVALID_ARG),
])
def test_sample_tokens_refusals(change, code):
    assert _sample(**change) == code


def test_sample_tokens_of_nothing():
    assert _sample(rows=0) == kap.OK


def _items(list_len=(40, 40, 50), n_q=(1, 4, 2), groups=(0, 2, 3), prefix=(30, 0), hq=32, hkv=8, **kw):
    return kap.shared_prefix_items(list_len, n_q, groups, prefix, hq, hkv, **kw)


@pytest.mark.parametrize("change,code", [
    (dict(list_len=(40, 0, 50)), kap.ERR_INVALID_ARG), (dict(n_q=(1, 0, 2)), kap.ERR_INVALID_ARG),
    (dict(groups=(0, 2, 2)), kap.ERR_INVALID_ARG), (dict(groups=(1, 2, 3)), kap.ERR_INVALID_ARG),
    (dict(groups=(0, 0, 3)), kap.ERR_INVALID_ARG), (dict(groups=(0, 4, 3)), kap.ERR_INVALID_ARG),
    (dict(prefix=(41, 0)), kap.ERR_INVALID_ARG), (dict(prefix=(-1, 0)), kap.ERR_INVALID_ARG),
    (dict(prefix=(30,)), kap.ERR_INVALID_ARG), (dict(n_q=(1, 4)), kap.ERR_INVALID_ARG),
    (dict(hq=30), kap.ERR_INVALID_ARG), (dict(hq=24), kap.ERR_UNSUPPORTED), (dict(hq=256), kap.ERR_UNSUPPORTED),
    (dict(n_q=(1, 17, 2)), kap.ERR_CAPACITY), (dict(max_rows_per_item=0), kap.ERR_INVALID_ARG), (dict(cta_slots=0), kap.ERR_INVALID_ARG),
])
def test_shared_prefix_refusals(change, code):
    with pytest.raises(kap.KapError) as e:
        _items(**change)
    assert e.value.code == code


def test_shared_prefix_items_of_good_groups():
    assert _items() >= 1
    assert kap.shared_prefix_items(np.array([1]), np.array([1]), np.array([0, 1]), np.array([0])) >= 1


def test_sample_tokens_refuses_rows_that_do_not_fit():
    most = 16 * 512 * 99
    assert _sample(vocab=most + 1, stride=most + 1) == kap.ERR_UNSUPPORTED
    assert b"vocab" in kap.lib().kap_last_error()
    assert _sample(vocab=100000, stride=100000, rows=0x7fffffff, k=A) == kap.ERR_UNSUPPORTED          # more CTAs than a grid has


def test_the_binding_refuses_host_tensors():
    import torch
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    rows = torch.zeros(2, 8, 128, dtype=bf)
    pool, idx, freq = torch.zeros(3, 2, 8, 16, 128, dtype=bf), torch.zeros(3, dtype=i32), torch.ones(64)
    with pytest.raises(kap.KapError, match="not on a GPU"):
        kap.append_kv_rope(None, rows, rows, pool, idx, idx, idx[:2], freq)
    with pytest.raises(kap.KapError, match="on cpu"):
        kap.sample_tokens(torch.zeros(2, 10), torch.zeros(2, dtype=f32), torch.zeros(2, dtype=i32))
