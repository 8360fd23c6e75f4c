"""Argument errors of the decoding calls that are found on the host: misaligned arrays, and sizes that would not fit the host's
memory or 32-bit indices.  The pointers are never followed."""

import pytest

from paper_2607_24260_b200 import kap
from test_host_decoding_ops import ODD, _append, _sample


@pytest.mark.parametrize("name", ["t", "k", "p", "m", "u", "token", "logprob"])
def test_sample_tokens_refuses_misaligned_arrays(name):
    assert _sample(**{name: ODD}) == kap.ERR_INVALID_ARG
    assert b"aligned" in kap.lib().kap_last_error()


@pytest.mark.parametrize("change", [dict(indptr=ODD), dict(freq=ODD), dict(pos=ODD, axes=1, pos_stride=4), dict(offset=ODD), dict(bti=ODD), dict(btp=ODD),
                                    dict(ctx=ODD), dict(status=ODD)])
def test_append_kv_rope_refuses_misaligned_arrays(change):
    assert _append(**change) == kap.ERR_INVALID_ARG
    assert b"aligned" in kap.lib().kap_last_error()
