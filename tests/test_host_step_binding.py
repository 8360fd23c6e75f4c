"""What the Python binding of the calls of a mixed step refuses before it hands pointers on, and what it hands on: tensors whose shapes, types, strides or
devices the kernels would misread.  The C entry points are replaced by ones that only note their arguments."""
import pytest
import torch

from paper_2607_24260_b200 import kap
from test_host_binding_checks import BF, F32, I32, I64, gpu, noted      # noqa: F401


class Workspace:
    device, kv_layout, _h = 0, kap.KV_HND, 77


def _refuses(f, **change):
    with pytest.raises(kap.KapError) as e:
        f(**change)
    assert e.value.code == kap.ERR_INVALID_ARG


def _chunk(**change):
    a = dict(q=gpu(9, 8, 128), q_indptr=gpu(4, dtype=I32), kv_pool=gpu(50, 2, 2, 16, 128), bt_indptr=gpu(4, dtype=I32), bt_pages=gpu(30, dtype=I32),
             ctx_len=gpu(3, dtype=I32), out=gpu(9, 8, 128), ws=Workspace(), lse=gpu(9, 8, dtype=F32), window=5, n_sink=2, stream=None)
    a.update(change)
    return kap.chunk_attn(**a)


@pytest.mark.parametrize("change", [
    dict(q=gpu(9, 8, 128, dtype=F32)), dict(q=gpu(9, 8, 128, index=1)), dict(q=gpu(9, 128, 8).transpose(1, 2)), dict(out=gpu(9, 8, 128, dtype=F32)),
    dict(out=gpu(8, 8, 128)), dict(out=gpu(9, 8, 128, index=1)), dict(lse=gpu(9, 8)), dict(lse=gpu(8, 8, dtype=F32)), dict(lse=gpu(8, 9, dtype=F32).transpose(0, 1)),
    dict(q_indptr=gpu(3, dtype=I32)), dict(q_indptr=gpu(4, dtype=I64)), dict(ctx_len=gpu(3, dtype=I64)), dict(bt_indptr=gpu(3, dtype=I32)),
    dict(bt_pages=gpu(30, dtype=I64)), dict(bt_pages=gpu(30, dtype=I32, index=1)), dict(kv_pool=gpu(50, 2, 2, 16, 64)), dict(kv_pool=gpu(50, 1, 2, 16, 128)),
    dict(kv_pool=gpu(50, 2, 2, 16, 128, dtype=F32)), dict(kv_pool=gpu(50, 2, 2, 128, 16).transpose(3, 4)),
])
def test_chunk_attn(change):
    _refuses(_chunk, **change)


def test_chunk_attn_hands_on(noted, monkeypatch):                       # noqa: F811
    monkeypatch.setattr(kap, "_stream_on", lambda dev, stream: 5)
    _chunk()
    name, args = noted[-1]
    assert name == "kap_chunk_attn" and args[2] == 9 and args[4] == 50 and args[8:13] == (3, 8, 2, 128, 16) and args[14:16] == (5, 2) and args[18:] == (77, 5)


def _build(**change):
    a = dict(ctx_len=gpu(3, dtype=I32), page_table=gpu(6, 10, dtype=I32), pages_held=gpu(6, dtype=I32), free_pages=gpu(40, dtype=I32), free_count=gpu(1, dtype=I32),
             bt_indptr=gpu(4, dtype=I32), bt_pages=gpu(30, dtype=I32), n_new=gpu(3, dtype=I32), request=gpu(3, dtype=I32), new_indptr=gpu(4, dtype=I32),
             slot=gpu(20, dtype=I64), position=gpu(25, dtype=I32), device_status=gpu(1, dtype=I32))
    a.update(change)
    return kap.build_block_tables(**a)


@pytest.mark.parametrize("change", [
    dict(ctx_len=gpu(3, dtype=I64)), dict(ctx_len=gpu(3, dtype=I32, index=1)), dict(page_table=gpu(60, dtype=I32)), dict(page_table=gpu(6, 10, dtype=I64)),
    dict(page_table=gpu(10, 6, dtype=I32).transpose(0, 1)), dict(pages_held=gpu(5, dtype=I32)), dict(pages_held=gpu(6, dtype=I64)), dict(free_pages=gpu(40, dtype=I64)),
    dict(free_count=gpu(0, dtype=I32)), dict(free_count=gpu(1, dtype=I64)), dict(bt_indptr=gpu(3, dtype=I32)), dict(bt_pages=gpu(30, dtype=I64)),
    dict(n_new=gpu(2, dtype=I32)), dict(request=gpu(3, dtype=I64)), dict(new_indptr=gpu(3, dtype=I32)), dict(slot=gpu(20, dtype=I32)), dict(position=gpu(20, dtype=I64)),
    dict(device_status=gpu(1, dtype=I64)), dict(free_pages=gpu(40, dtype=I32, index=1)),
])
def test_build_block_tables(change):
    _refuses(_build, **change)


def test_build_block_tables_hands_on(noted, monkeypatch):               # noqa: F811
    monkeypatch.setattr(kap, "_stream_on", lambda dev, stream: 5)
    _build()
    name, args = noted[-1]
    assert name == "kap_build_block_tables" and args[3:5] == (3, 16) and args[6:8] == (6, 10) and args[10] == 40 and args[14] == 30 and args[18] == 20
    _build(slot=None)
    assert noted[-1][1][16] is None and noted[-1][1][18] == 25
    _build(slot=None, position=None, new_indptr=None, n_new=None, request=None, device_status=None)
    assert noted[-1][1][15:20] == (None, None, None, 0, None)


@pytest.mark.parametrize("change", [
    dict(request=gpu(3, dtype=I64)), dict(keep_tokens=gpu(2, dtype=I32)), dict(keep_tokens=gpu(3, dtype=I64)), dict(pages_held=gpu(5, dtype=I32)),
    dict(device_status=gpu(0, dtype=I32)),
])
def test_release_pages(change):
    a = dict(request=gpu(3, dtype=I32), page_table=gpu(6, 10, dtype=I32), pages_held=gpu(6, dtype=I32), free_pages=gpu(40, dtype=I32), free_count=gpu(1, dtype=I32),
             keep_tokens=gpu(3, dtype=I32), device_status=gpu(1, dtype=I32))
    _refuses(kap.release_pages, **{**a, **change})


def _append(**change):
    a = dict(q=gpu(9, 8, 128), k_new=gpu(9, 2, 128), v_new=gpu(9, 2, 128), kv_pool=gpu(50, 2, 2, 16, 128), bt_indptr=gpu(4, dtype=I32), bt_pages=gpu(30, dtype=I32),
             ctx_len=gpu(3, dtype=I32), inv_freq=gpu(64, dtype=F32), q_weight=gpu(128), k_weight=gpu(128), new_indptr=gpu(4, dtype=I32))
    a.update(change)
    return kap.append_kv_norm_rope(**a)


@pytest.mark.parametrize("change", [
    dict(q_weight=gpu(64)), dict(q_weight=gpu(7, 128)), dict(q_weight=gpu(8, 128)), dict(q_weight=gpu(128, dtype=F32)), dict(q_weight=gpu(128, dtype=I32), k_weight=gpu(128, dtype=I32)),
    dict(k_weight=gpu(128, index=1)), dict(k_weight=gpu(8, 128)), dict(q_weight=gpu(128, 8).transpose(0, 1), k_weight=gpu(2, 128)), dict(k_new=gpu(9, 2, 64)),
    dict(inv_freq=gpu(64)), dict(new_indptr=gpu(3, dtype=I32)),
])
def test_append_kv_norm_rope(change):
    _refuses(_append, **change)


def test_append_kv_norm_rope_hands_on(noted, monkeypatch):              # noqa: F811
    monkeypatch.setattr(kap, "_stream_on", lambda dev, stream: 5)
    for change, want in ((dict(), (kap.NORM_BF16, 0, 0, 1e-6)), (dict(q_weight=gpu(8, 128, dtype=F32), k_weight=gpu(2, 128, dtype=F32), unit_offset=True, eps=0.5), (kap.NORM_F32, 1, 1, 0.5)),
                         (dict(q_weight=None, k_weight=None), (kap.NORM_F32, 0, 0, 1e-6))):
        _append(**change)
        name, args = noted[-1]
        assert name == "kap_append_kv_norm_rope" and args[12:16] == want
    kap.append_kv_rope(gpu(9, 8, 128), gpu(9, 2, 128), gpu(9, 2, 128), gpu(50, 2, 2, 16, 128), gpu(4, dtype=I32), gpu(30, dtype=I32), gpu(3, dtype=I32), gpu(64, dtype=F32),
                       new_indptr=gpu(4, dtype=I32))
    assert noted[-1][0] == "kap_append_kv_rope" and len(noted[-1][1]) == 32


def _logits(**change):
    a = dict(logits=gpu(3, 100, dtype=F32), out=gpu(3, 100, dtype=F32), history=gpu(50, dtype=I32), history_at=gpu(3, 3, dtype=I64), repetition=gpu(3, dtype=F32),
             presence=gpu(3, dtype=F32), frequency=gpu(3, dtype=F32), bias_indptr=gpu(4, dtype=I32), bias_token=gpu(7, dtype=I32), bias_value=gpu(7, dtype=F32),
             allowed=gpu(2, 4, dtype=I32), allowed_row=gpu(3, dtype=I32))
    a.update(change)
    return kap.adjust_logits(**a)


@pytest.mark.parametrize("change", [
    dict(logits=gpu(3, 100, dtype=I32)), dict(logits=gpu(100, dtype=F32)), dict(logits=gpu(100, 3, dtype=F32).transpose(0, 1)), dict(out=gpu(3, 100)),
    dict(out=gpu(3, 99, dtype=F32)), dict(out=gpu(3, 100, dtype=F32, index=1)), dict(history=gpu(50, dtype=I64)), dict(history_at=gpu(3, 3, dtype=I32)),
    dict(history_at=gpu(2, 3, dtype=I64)), dict(repetition=gpu(2, dtype=F32)), dict(presence=gpu(3)), dict(frequency=gpu(3, dtype=F32, index=1)), dict(bias_indptr=gpu(3, dtype=I32)),
    dict(bias_token=gpu(7, dtype=I64)), dict(bias_value=gpu(6, dtype=F32)), dict(allowed=gpu(2, 3, dtype=I32)), dict(allowed=gpu(4, 2, dtype=I32).transpose(0, 1)),
    dict(allowed=gpu(2, 4, dtype=I64)), dict(allowed_row=gpu(2, dtype=I32)),
])
def test_adjust_logits(change):
    _refuses(_logits, **change)


def test_adjust_logits_hands_on(noted, monkeypatch):                    # noqa: F811
    monkeypatch.setattr(kap, "_stream_on", lambda dev, stream: 5)
    _logits(logits=gpu(3, 105, dtype=F32)[:, :100])
    name, args = noted[-1]
    assert name == "kap_adjust_logits" and args[1:5] == (kap.LOGITS_F32, 105, 3, 100) and args[6] == 100 and args[8] == 50 and args[16] == 7 and args[18:20] == (2, 4)
    _logits(out=None)
    assert noted[-1][1][0] == noted[-1][1][5]
