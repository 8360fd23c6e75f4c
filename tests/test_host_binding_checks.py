"""What the Python binding refuses before it hands pointers on: tensors whose shapes, types, strides or devices the kernels would
misread.  Nothing is launched: the tensors here only say that they are on a GPU and have addresses that nobody follows."""
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


def passes_the_binding(call):
    """the C entry point answers: here with an error of its own, since there is neither a workspace nor a GPU"""
    with pytest.raises(kap.KapError) as e:
        call()
    return "NULL workspace" in str(e.value)


def test_shared_prefix_attn_takes_the_scheduled_rows_and_more():
    assert passes_the_binding(attend)
    assert passes_the_binding(lambda: attend(rows=11))
    assert passes_the_binding(lambda: attend(q=gpu(11, 8, 128), lse=None))


@pytest.mark.parametrize("change", [
    dict(rows=2), dict(rows=7), dict(q=gpu(7, 8, 128)), dict(out=gpu(7, 8, 128)), dict(lse=gpu(7, 8, dtype=F32)), dict(lse=gpu(8, 7, dtype=F32)),
    dict(out=gpu(8, 4, 128)), dict(out=gpu(8, 8, 64)), dict(ws=Scheduled(9)),
])
def test_shared_prefix_attn_refuses_arrays_with_fewer_rows_than_scheduled(change):
    with pytest.raises(kap.KapError, match="scheduled rows") as e:
        attend(**change)
    assert e.value.code == kap.ERR_INVALID_ARG
