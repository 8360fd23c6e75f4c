"""What the Python binding refuses before it hands pointers on: tensors whose shapes, types, strides or devices the kernels would
misread.  The C entry points are replaced by ones that only note their arguments, and the tensors here only say that they are on a GPU."""
import pytest
import torch

from paper_2607_24260_b200 import kap

BF, F32, I32, I64 = torch.bfloat16, torch.float32, torch.int32, torch.int64


class OnGpu:
    """a tensor's shape, type and strides, on device `index`"""

    def __init__(self, t, index=0):
        self.t, self.index = t, index
        self.dtype, self.is_cuda, self.device = t.dtype, True, torch.device("cuda", index)

    shape = property(lambda self: self.t.shape)

    def __getitem__(self, i):
        return OnGpu(self.t[i], self.index)

    def view(self, *shape):
        return OnGpu(self.t.view(*shape), self.index)

    def transpose(self, a, b):
        return OnGpu(self.t.transpose(a, b), self.index)

    def data_ptr(self):
        return (1 << 30) + self.t.storage_offset() * self.t.element_size()

    def get_device(self):
        return self.index

    def __getattr__(self, name):
        return getattr(self.t, name)


def gpu(*shape, dtype=BF, index=0):
    return OnGpu(torch.empty(shape, dtype=dtype, device="meta"), index)


@pytest.fixture(autouse=True)
def noted(monkeypatch):
    """the arguments of the C calls that the binding makes"""
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: calls.append((name, args)) or kap.OK

    monkeypatch.setattr(kap, "_lib", Library())
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return calls


class Scheduled:
    """a workspace that holds a shared-prefix schedule of so many rows"""

    def __init__(self, rows, kv_layout=kap.KV_HND):
        self.shared_prefix_rows, self.kv_layout, self._h, self.device = rows, kv_layout, None, 0


STREAM = type("Stream", (), dict(cuda_stream=None))()


def attend(rows=8, hq=8, hkv=2, batch=2, **change):
    a = dict(q=gpu(rows, hq, 128), q_indptr=gpu(batch + 1, dtype=I32), kv_pool=gpu(9, 2, hkv, 16, 128), bt_indptr=gpu(batch + 1, dtype=I32),
             bt_pages=gpu(12, dtype=I32), ctx_len=gpu(batch, dtype=I32), out=gpu(rows, hq, 128), ws=Scheduled(8), lse=gpu(rows, hq, dtype=F32),
             stream=STREAM)
    assert set(change) <= set(a) | {"sm_scale"}
    a.update(change)
    kap.shared_prefix_attn(**a)


def refused(noted, match, call, **change):
    with pytest.raises(kap.KapError, match=match) as e:
        call(**change)
    assert e.value.code == kap.ERR_INVALID_ARG and not noted


def test_shared_prefix_attn_takes_the_scheduled_rows_and_more(noted):
    attend()
    attend(rows=11)
    attend(q=gpu(11, 8, 128), lse=None)
    assert [name for name, _ in noted] == ["kap_shared_prefix_attn"] * 3


@pytest.mark.parametrize("change", [
    dict(rows=2), dict(rows=7), dict(q=gpu(7, 8, 128)), dict(out=gpu(7, 8, 128)), dict(lse=gpu(7, 8, dtype=F32)), dict(lse=gpu(8, 7, dtype=F32)),
    dict(out=gpu(8, 4, 128)), dict(out=gpu(8, 8, 64)), dict(ws=Scheduled(9)),
])
def test_shared_prefix_attn_refuses_arrays_with_fewer_rows_than_scheduled(noted, change):
    refused(noted, "scheduled rows", attend, **change)


def append(rows=4, hq=8, hkv=2, batch=4, d=128, **change):
    a = dict(q=gpu(rows, hq, d), k_new=gpu(rows, hkv, d), v_new=gpu(rows, hkv, d), kv_pool=gpu(9, 2, hkv, 16, 128), bt_indptr=gpu(batch + 1, dtype=I32),
             bt_pages=gpu(12, dtype=I32), ctx_len=gpu(batch, dtype=I32), inv_freq=gpu(64, dtype=F32), q_out=gpu(rows, hq, d), stream=STREAM)
    assert set(change) <= set(a) | {"new_indptr", "positions", "freq_axis", "position_offset", "device_status", "kv_layout"}
    a.update(change)
    kap.append_kv_rope(**a)


def test_append_kv_rope_passes_views_of_a_fused_projection_on(noted):
    fused = gpu(4, 12, 128)
    append(q=fused[:, :8], k_new=fused[:, 8:10], v_new=fused[:, 10:], q_out=None)
    append(q=None)
    append(kv_pool=gpu(9, 2, 16, 2, 128), kv_layout=kap.KV_NHD)
    strides = noted[0][1]
    assert (strides[1], strides[3], strides[5], strides[7]) == (12 * 128,) * 4 and strides[6] == strides[0]
    assert len(noted) == 3


@pytest.mark.parametrize("change", [
    # heads of 64 columns whose rows are far enough apart for two heads of 128
    dict(k_new=gpu(4, 32, 64)[:, 16:18], v_new=gpu(4, 32, 64)[:, 18:20]), dict(k_new=gpu(4, 32, 64)[:, 16:18]), dict(v_new=gpu(4, 32, 64)[:, 16:18]),
    dict(q=gpu(4, 32, 64)[:, :8]), dict(q=gpu(4, 32, 64)[:, :8], q_out=None), dict(q_out=gpu(4, 32, 64)[:, :8]), dict(d=64), dict(d=256),
])
def test_append_kv_rope_refuses_heads_of_another_width_than_the_pools(noted, change):
    refused(noted, "expected bfloat16", append, **change)


@pytest.mark.parametrize("change", [
    dict(bt_indptr=gpu(5, dtype=I64)), dict(bt_pages=gpu(12, dtype=I64)), dict(ctx_len=gpu(4, dtype=I64)), dict(ctx_len=gpu(4, dtype=F32)),
    dict(bt_pages=gpu(24, dtype=I32)[::2]), dict(bt_indptr=gpu(10, dtype=I32)[::2]), dict(ctx_len=gpu(4, 2, dtype=I32)[:, 0]),
    dict(bt_indptr=gpu(4, dtype=I32)), dict(new_indptr=gpu(5, dtype=I64)), dict(new_indptr=gpu(4, dtype=I32)), dict(new_indptr=gpu(10, dtype=I32)[::2]),
    dict(position_offset=gpu(4, dtype=I64)), dict(position_offset=gpu(3, dtype=I32)), dict(position_offset=gpu(4, dtype=F32)),
    dict(device_status=gpu(1, dtype=I64)), dict(device_status=gpu(0, dtype=I32)),
])
def test_append_kv_rope_refuses_index_arrays_that_it_would_misread(noted, change):
    refused(noted, "contiguous int32", append, **change)


def test_append_kv_rope_takes_longer_index_arrays(noted):
    append(bt_indptr=gpu(9, dtype=I32), new_indptr=gpu(9, dtype=I32), position_offset=gpu(9, dtype=I32), device_status=gpu(2, dtype=I32))
    append(new_indptr=gpu(5, dtype=I32), position_offset=gpu(4, dtype=I32), device_status=gpu(1, dtype=I32))
    assert len(noted) == 2


@pytest.mark.parametrize("change", [
    dict(kv_pool=gpu(9, 2, 2, 16, 128, dtype=torch.float16)), dict(kv_pool=gpu(9, 2, 2, 16, 128, dtype=F32)),
    dict(kv_pool=gpu(9, 2, 16, 2, 128).transpose(2, 3)), dict(kv_pool=gpu(18, 2, 2, 16, 128)[::2]), dict(kv_pool=gpu(9, 3, 2, 16, 128)[:, :2]),
    dict(kv_pool=gpu(9, 1, 2, 16, 128)), dict(kv_pool=gpu(9, 3, 2, 16, 128)),
])
def test_append_kv_rope_refuses_pools_that_are_not_dense_bf16(noted, change):
    refused(noted, "kv_pool", append, **change)


@pytest.mark.parametrize("change,match", [
    (dict(q=gpu(8, 8, 128, dtype=torch.float16)), "bfloat16"), (dict(q=gpu(8, 8, 128, dtype=F32)), "bfloat16"), (dict(out=gpu(8, 8, 128, dtype=F32)), "bfloat16"),
    (dict(q=gpu(8, 12, 128)[:, :8]), "contiguous"), (dict(q=gpu(16, 8, 128)[::2]), "contiguous"), (dict(out=gpu(8, 8, 256)[..., :128]), "contiguous"),
    (dict(q=gpu(8, 8, 128).transpose(0, 1)), "contiguous"), (dict(lse=gpu(8, 8)), "lse"), (dict(lse=gpu(8, 8, dtype=F32).transpose(0, 1)), "lse"),
    (dict(kv_pool=gpu(9, 2, 2, 16, 128, dtype=torch.float16)), "kv_pool"), (dict(kv_pool=gpu(9, 2, 16, 2, 128).transpose(2, 3)), "kv_pool"),
    (dict(kv_pool=gpu(18, 2, 2, 16, 128)[::2]), "kv_pool"), (dict(kv_pool=gpu(9, 2, 2, 16, 64)), "kv_pool"),
    (dict(q_indptr=gpu(3, dtype=I64)), "q_indptr"), (dict(q_indptr=gpu(2, dtype=I32)), "q_indptr"), (dict(bt_indptr=gpu(3, dtype=I64)), "bt_indptr"),
    (dict(bt_indptr=gpu(2, dtype=I32)), "bt_indptr"), (dict(bt_pages=gpu(12, dtype=I64)), "bt_pages"), (dict(bt_pages=gpu(24, dtype=I32)[::2]), "bt_pages"),
    (dict(ctx_len=gpu(2, dtype=I64)), "ctx_len"), (dict(ctx_len=gpu(4, dtype=I32)[::2]), "ctx_len"),
])
def test_shared_prefix_attn_refuses_arrays_that_it_would_misread(noted, change, match):
    refused(noted, match, attend, **change)


def test_shared_prefix_attn_takes_pools_of_either_layout(noted):
    attend(kv_pool=gpu(9, 2, 16, 2, 128), ws=Scheduled(8, kap.KV_NHD))
    attend(q_indptr=gpu(9, dtype=I32), bt_indptr=gpu(9, dtype=I32))
    assert len(noted) == 2


def sample(rows=4, vocab=50, **change):
    f = lambda dtype=F32: gpu(rows, dtype=dtype)                                  # noqa: E731
    a = dict(logits=gpu(rows, vocab, dtype=F32), uniform=f(), token=f(I32), logprob=f(), temperature=f(), top_k=f(I32), top_p=f(), min_p=f(), stream=STREAM)
    assert set(change) <= set(a)
    a.update(change)
    kap.sample_tokens(**a)


APPEND = dict(q=(4, 8, 128), k_new=(4, 2, 128), v_new=(4, 2, 128), kv_pool=(9, 2, 2, 16, 128), bt_indptr=(5, I32), bt_pages=(12, I32), ctx_len=(4, I32),
              inv_freq=(64, F32), q_out=(4, 8, 128), new_indptr=(5, I32), positions=(4, I32), device_status=(1, I32))
OFFSET = dict(position_offset=(4, I32))
ATTEND = dict(q=(8, 8, 128), q_indptr=(3, I32), kv_pool=(9, 2, 2, 16, 128), bt_indptr=(3, I32), bt_pages=(12, I32), ctx_len=(2, I32), out=(8, 8, 128), lse=(8, 8, F32))
SAMPLE = dict(logits=(4, 50, F32), uniform=(4, F32), token=(4, I32), logprob=(4, F32), temperature=(4, F32), top_k=(4, I32), top_p=(4, F32), min_p=(4, F32))


def shape_type(s):
    return (s[:-1], s[-1]) if isinstance(s[-1], torch.dtype) else (s, BF)


EACH = [(call, name, shape) for call, arrays in ((append, APPEND), (append, OFFSET), (attend, ATTEND), (sample, SAMPLE)) for name, shape in arrays.items()]


@pytest.mark.parametrize("call,name,shape", EACH, ids=lambda x: x if isinstance(x, str) else getattr(x, "__name__", ""))
def test_an_array_on_another_device_than_the_others_is_refused(noted, call, name, shape):
    size, dtype = shape_type(shape)
    refused(noted, "GPU|device", call, **{name: gpu(*size, dtype=dtype, index=1)})
    refused(noted, "GPU|on cpu", call, **{name: torch.empty(size, dtype=dtype)})  # in host memory


@pytest.mark.parametrize("call,arrays", [(append, APPEND), (attend, ATTEND), (sample, SAMPLE)], ids=["append", "attend", "sample"])
def test_arrays_on_another_device_than_the_current_one_are_refused(noted, monkeypatch, call, arrays):
    there = {}
    for name, shape in arrays.items():
        size, dtype = shape_type(shape)
        there[name] = gpu(*size, dtype=dtype, index=1)
    refused(noted, "device", call, **there)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    if call is attend:                                                            # the workspace is on device 0
        refused(noted, "device", call, **there)
        there["ws"] = Scheduled(8)
        there["ws"].device = 1
    call(**there)
    assert len(noted) == 1


def test_the_current_stream_is_found_without_the_short_way_too(monkeypatch):
    class Torch:
        _C = object()

        class cuda:
            @staticmethod
            def current_stream(dev):
                return type("Stream", (), dict(cuda_stream=1000 + dev))()

    assert kap._stream_reader(Torch)(3) == 1003
