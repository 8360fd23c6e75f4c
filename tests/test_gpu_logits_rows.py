"""kap_adjust_logits on the GPU: offsets are checked in every row, and what no rule names stays bit for bit."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap
from test_gpu_adjust_logits import BF16, F32, Case

pytestmark = pytest.mark.gpu
BIT = 1 << kap.ERR_DEVICE_INDEX
BAD = [[-1, 0, 5], [5, 4, 9], [0, 9, 4], [0, 1, 10 ** 9], [2 ** 62, 2 ** 62, 2 ** 62]]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("bad", BAD)
def test_offsets_of_a_row_without_penalties_are_checked(bad, in_place):
    c = Case(60, 4, 300, masks=2)
    c.rep[2], c.pres[2], c.freq[2] = 1.0, 0.0, 0.0
    c.at[2] = bad
    out, a = c.run(in_place=in_place)
    c.at[2] = 0
    c.check(out, a, BIT)
    # switched off by what is no parameter
    c.status.zero_()
    c.rep[2], c.pres[2], c.freq[2] = np.nan, np.nan, np.nan
    c.at[2] = bad
    out, a = c.run(in_place=in_place)
    c.at[2] = 0
    c.check(out, a, BIT)


@pytest.mark.parametrize("bad", BAD)
def test_offsets_of_a_call_without_penalties_are_checked(bad):
    c = Case(61, 4, 300, masks=2)
    for at, status in ((c.at[1].copy(), 0), (bad, BIT)):
        c.status.zero_()
        c.at[1] = at
        out, a = c.run(drop=("repetition", "presence", "frequency"))
        c.check(out, {k: v for k, v in a.items() if k != "history"}, status)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,pad,out_pad", [(F32, 0, 0), (F32, 1, 2), (BF16, 0, 0), (BF16, 1, 8)])
@pytest.mark.parametrize("vocab", [7, 1000, 50257])
def test_what_no_rule_names_is_the_logit_itself(vocab, dtype, pad, out_pad, in_place):
    c = Case(vocab + 1, 6, vocab, dtype, pad, out_pad, longest=max(3, vocab // 10), masks=3)
    # among them values that arithmetic would change
    c.logits[:, ::3] = float("nan")
    c.logits[:, 1::5] = 1e-41
    c.logits[:, 2::7] = -0.0
    out, a = c.run(in_place=in_place)
    torch.cuda.synchronize()
    bits = torch.int32 if dtype is F32 else torch.int16
    same = (out.contiguous().view(bits) == c.logits.contiguous().view(bits)).cpu().numpy()
    for r in range(c.rows):
        named = np.zeros(vocab, dtype=bool)
        b, _, e = c.at[r]
        t = c.history[b:e]
        named[t[(t >= 0) & (t < vocab)]] = True
        named[c.bias_token[c.bias_at[r]:c.bias_at[r + 1]]] = True
        if c.mask_row[r] >= 0:
            named |= np.unpackbits(c.masks[c.mask_row[r]].view(np.uint8), bitorder="little")[:vocab] == 0
        assert same[r][~named].all()
        assert vocab < 100 or not named.all()
