"""Refusals of kap_chunk_attn_items, kap_append_kv_norm_rope, kap_build_block_tables, kap_release_pages and kap_adjust_logits: argument
errors are found on the host before anything is launched, so they can be seen without a GPU (the pointers are never followed)."""
import ctypes as C

import pytest

from paper_2607_24260_b200 import kap

A = C.c_void_p(1 << 20)                        # an aligned address that nothing reads
ODD, HALF = C.c_void_p((1 << 20) + 2), C.c_void_p((1 << 20) + 4)
INVALID, UNSUPPORTED = kap.ERR_INVALID_ARG, kap.ERR_UNSUPPORTED


def _call(name, defaults, change):
    assert set(change) <= set(defaults)
    return getattr(kap.lib(), name)(*{**defaults, **change}.values())


APPEND = dict(q=A, qs=4096, k=A, ks=1024, v=A, vs=1024, qo=A, qos=4096, indptr=None, rows=4, qw=A, kw=A, kind=0, per_head=0, unit=0, eps=1e-6, freq=A, rot=128,
              inter=0, pos=None, pos_stride=0, axes=0, axis=None, offset=None, pool=A, pages=10, bti=A, btp=A, ctx=A, advance=1, batch=4, hq=32, hkv=8,
              d=128, page=16, layout=0, status=None, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(kind=2), UNSUPPORTED), (dict(kind=-1), UNSUPPORTED), (dict(eps=-1e-9), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(qw=HALF), INVALID), (dict(kw=ODD), INVALID), (dict(d=64), UNSUPPORTED), (dict(rot=24), UNSUPPORTED), (dict(rows=5), INVALID), (dict(k=None), INVALID),
    (dict(qo=None), INVALID), (dict(ks=1016), INVALID), (dict(axes=2), INVALID), (dict(layout=2), INVALID), (dict(ctx=ODD), INVALID),
])
def test_append_kv_norm_rope_refusals(change, code):
    assert _call("kap_append_kv_norm_rope", APPEND, change) == code
    assert kap.lib().kap_last_error()


def test_append_kv_norm_rope_of_nothing():
    assert _call("kap_append_kv_norm_rope", APPEND, dict(batch=0, rows=0)) == kap.OK
    assert _call("kap_append_kv_norm_rope", APPEND, dict(rows=0, indptr=A)) == kap.OK


BUILD = dict(request=A, ctx=A, new=A, batch=4, page=16, table=A, requests=8, stride=10, held=A, free=A, capacity=100, count=A, bti=A, btp=A, bt_capacity=40, indptr=A,
             slot=A, position=A, rows=100, status=None, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(batch=-1), INVALID), (dict(batch=9), INVALID), (dict(page=0), INVALID), (dict(page=-16), INVALID), (dict(requests=-1), INVALID), (dict(stride=-1), INVALID),
    (dict(capacity=-1), INVALID), (dict(bt_capacity=-1), INVALID), (dict(rows=-1), INVALID), (dict(table=None), INVALID), (dict(held=None), INVALID),
    (dict(free=None), INVALID), (dict(count=None), INVALID), (dict(ctx=None), INVALID), (dict(bti=None), INVALID), (dict(btp=None), INVALID), (dict(indptr=None), INVALID),
    (dict(slot=HALF), INVALID), (dict(position=ODD), INVALID), (dict(request=ODD), INVALID), (dict(new=ODD), INVALID), (dict(table=ODD), INVALID), (dict(status=ODD), INVALID),
    (dict(requests=2 ** 20 + 1), UNSUPPORTED), (dict(stride=2 ** 31), UNSUPPORTED),
])
def test_build_block_tables_refusals(change, code):
    assert _call("kap_build_block_tables", BUILD, change) == code
    assert kap.lib().kap_last_error()


RELEASE = dict(request=A, n=4, keep=A, page=16, table=A, requests=8, stride=10, held=A, free=A, capacity=100, count=A, status=None, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(n=-1), INVALID), (dict(n=9), INVALID), (dict(page=0), INVALID), (dict(table=None), INVALID), (dict(held=None), INVALID), (dict(free=None), INVALID),
    (dict(count=None), INVALID), (dict(keep=ODD), INVALID), (dict(request=ODD), INVALID), (dict(requests=2 ** 20 + 1), UNSUPPORTED),
])
def test_release_pages_refusals(change, code):
    assert _call("kap_release_pages", RELEASE, change) == code


def test_release_of_nothing():
    assert _call("kap_release_pages", RELEASE, dict(n=0)) == kap.OK


LOGITS = dict(logits=A, kind=0, stride=100, rows=2, vocab=100, out=A, out_stride=100, history=A, history_len=50, at=A, rep=A, pres=A, freq=A, bias_at=A, bias_token=A,
              bias_value=A, bias_len=5, allowed=A, masks=3, words=4, row=A, status=None, stream=None)


@pytest.mark.parametrize("change,code", [
    (dict(kind=2), UNSUPPORTED), (dict(kind=-1), UNSUPPORTED), (dict(rows=-1), INVALID), (dict(rows=65536), UNSUPPORTED), (dict(vocab=0), INVALID),
    (dict(vocab=811009, stride=811009, out_stride=811009), UNSUPPORTED), (dict(stride=99), INVALID), (dict(out_stride=99), INVALID), (dict(out_stride=104), INVALID),
    (dict(logits=None), INVALID), (dict(out=None), INVALID), (dict(logits=ODD), INVALID), (dict(logits=C.c_void_p((1 << 20) + 1), kind=1), INVALID),
    (dict(at=None), INVALID), (dict(history=None), INVALID), (dict(history_len=-1), INVALID), (dict(bias_at=None), INVALID), (dict(bias_token=None), INVALID),
    (dict(bias_value=None), INVALID), (dict(bias_len=-1), INVALID), (dict(masks=0), INVALID), (dict(words=3), INVALID), (dict(allowed=None), INVALID),
    (dict(row=None, masks=1), INVALID), (dict(at=HALF), INVALID), (dict(rep=ODD), INVALID), (dict(allowed=ODD), INVALID), (dict(bias_value=ODD), INVALID),
])
def test_adjust_logits_refusals(change, code):
    assert _call("kap_adjust_logits", LOGITS, change) == code
    assert kap.lib().kap_last_error()


@pytest.mark.parametrize("change", [dict(history=None, history_len=0, at=None), dict(bias_at=None, bias_token=None, bias_value=None), dict(bias_token=None, bias_value=None, bias_len=5),
                                    dict(bias_at=None, bias_len=0)])
def test_adjust_logits_refuses_half_a_rule(change):
    assert _call("kap_adjust_logits", LOGITS, change) == INVALID


def test_adjust_logits_of_nothing():
    assert _call("kap_adjust_logits", LOGITS, dict(rows=0)) == kap.OK


def test_chunk_attn_items():
    # four states of 256 rows for each of 148 SMs and how the work was divided, in items of 64 or of 5 rows
    rows = 4 * 148 * 256
    assert rows < kap.chunk_attn_items(64, 148) * 64 < rows + 64 * 2
    assert rows < kap.chunk_attn_items(5, 148) * 5 < rows + 20
    assert kap.chunk_attn_items() == kap.chunk_attn_items(64, 148)
    for bad in ((0, 148), (65, 148), (64, 0), (64, 5000)):
        with pytest.raises(kap.KapError) as e:
            kap.chunk_attn_items(*bad)
        assert e.value.code == INVALID
    assert kap.lib().kap_chunk_attn_items(64, 148, None) == INVALID


def test_chunk_attn_needs_a_workspace():
    args = [A, A, 4, A, 10, A, A, A, 1, 8, 2, 128, 16, C.c_float(0.1), 0, 0, A, None, None, None]
    assert kap.lib().kap_chunk_attn(*args) == INVALID
