"""Argument errors of the decoding calls that are found on the host: misaligned arrays, and sizes that would not fit the host's
memory or 32-bit indices.  The pointers are never followed."""
import numpy as np
import pytest

from paper_2607_24260_b200 import kap
from test_host_decoding_ops import ODD, _append, _items, _sample


@pytest.mark.parametrize("name", ["t", "k", "p", "m", "u", "token", "logprob"])
def test_sample_tokens_refuses_misaligned_arrays(name):
    assert _sample(**{name: ODD}) == kap.ERR_INVALID_ARG
    assert b"aligned" in kap.lib().kap_last_error()


@pytest.mark.parametrize("change", [dict(indptr=ODD), dict(freq=ODD), dict(pos=ODD, axes=1, pos_stride=4), dict(offset=ODD), dict(bti=ODD), dict(btp=ODD),
                                    dict(ctx=ODD), dict(status=ODD)])
def test_append_kv_rope_refuses_misaligned_arrays(change):
    assert _append(**change) == kap.ERR_INVALID_ARG
    assert b"aligned" in kap.lib().kap_last_error()


@pytest.mark.parametrize("slots", [4097, 2 ** 31 - 1])
def test_shared_prefix_items_refuses_devices_that_there_are_not(slots):
    with pytest.raises(kap.KapError) as e:
        _items(cta_slots=slots)
    assert e.value.code == kap.ERR_INVALID_ARG
    assert _items(cta_slots=4096) >= 1


def test_shared_prefix_items_refuses_more_lists_than_it_indexes():
    with pytest.raises(kap.KapError) as e:
        _items(hq=2 ** 30, hkv=2 ** 30)                                          # would be 3 x 2^30 units
    assert e.value.code == kap.ERR_CAPACITY
    n = 1 << 20
    with pytest.raises(kap.KapError) as e:
        kap.shared_prefix_items(np.full(n, 2), np.full(n, 1), np.array([0, n]), np.array([1]), 1024, 64)
    assert e.value.code == kap.ERR_CAPACITY


def test_shared_prefix_items_of_many_sequences():
    n = 8000
    assert kap.shared_prefix_items(np.full(n, 9), np.full(n, 1), np.array([0, n]), np.array([5]), 8, 2) >= n // 8
