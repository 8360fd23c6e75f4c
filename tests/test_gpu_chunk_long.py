"""kap_chunk_attn on the GPU over contexts so long that the order of the sums counts, against 64 bits.

The block tables name a few pages again and again, so a context of any length has few different tokens, and its softmax is a sum over them with their
multiplicities.  Tolerance: the sum l of a row's weights is a tree of fp32 sums no deeper than the 22 of a step's 80 weights, 2048 steps, and one for each
further 2048 steps or state that joins (at most 410 for the longest context, and 148 states): 2^-24 each, below 2^-24 2700 = 1.7e-4 of l, so much for lse too; scores are fp32 sums of
128 products and 2e-5 of lse as in the other tests.  The result's sum takes five products a step, each of which may cut off up to 2^-23 of the value
(the tensor core's rounding is not documented): 2^-23 5 2048 = 1.3e-3, and the further steps 1.7e-4; the weights are rounded to bf16 in front (2^-8 of the weighted mean of |V|), the result
once (2^-8 of it)."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap

pytestmark = pytest.mark.gpu
D, PAGE = 128, 16
LSE = 2.0 ** -24 * 2700 + 2e-5
SUM = 2.0 ** -23 * 5 * 2048 + 2.0 ** -24 * 2700


def _ws(batch, layout=kap.KV_HND):
    ws = kap.Workspace(max_items=kap.chunk_attn_items(), max_rows_per_item=64, max_batch=batch)
    ws.set_kv_layout(layout)
    return ws


@pytest.mark.parametrize("n", [1, 129])
def test_equal_weights_that_are_no_powers_of_two(n):
    """a first token with weight 1 and 2^24 others with e^-1, in units that a CTA does whole: a sum kept in one number would lose what is small beside it"""
    batch, tokens = 148, 2 ** 24
    pool = torch.zeros((2, 2, 1, PAGE, D), dtype=torch.bfloat16, device=gu.DEV)
    pool[:, 0, :, :, 0] = -1.0
    pool[0, 0, :, 0, 0] = 0.0
    value = (1 + torch.arange(D, device=gu.DEV) % 7).to(torch.bfloat16)
    pool[:, 1] = value
    pool[0, 1, :, 0] = 0.0
    pages = tokens // PAGE
    table = torch.ones((batch, pages), dtype=torch.int32, device=gu.DEV)
    table[:, 0] = 0
    q = torch.zeros((batch * n, 1, D), dtype=torch.bfloat16, device=gu.DEV)
    q[:, :, 0] = 1.0
    out, lse = torch.full_like(q, float("nan")), torch.full((batch * n, 1), float("nan"), device=gu.DEV)
    ws = _ws(batch)
    kap.chunk_attn(q, gu.i32(np.arange(batch + 1) * n), pool, gu.i32(np.arange(batch + 1) * pages), table.view(-1), gu.i32([tokens] * batch), out, ws, lse=lse, sm_scale=1.0)
    ws.check()
    others = tokens - n + torch.arange(n, device=gu.DEV, dtype=torch.float64)
    l = 1 + others * np.exp(-1.0)
    assert float((lse.view(batch, n).double() - l.log()).abs().max()) <= LSE
    ref = (others * np.exp(-1.0) / l)[:, None] * value.double()
    assert bool(((out.view(batch, n, D).double() - ref).abs() <= (2 * 2.0 ** -8 + SUM) * ref).all())


def test_units_of_the_longest_context():
    # two tiles over 2^26 tokens, by one CTA each: seconds, in which no wait may run out
    batch, n, tokens = 148, 129, 2 ** 26
    pool = torch.zeros((2, 2, 1, PAGE, D), dtype=torch.bfloat16, device=gu.DEV)
    value = (1 + torch.arange(D, device=gu.DEV) % 7).to(torch.bfloat16)
    pool[1, 1] = value
    pages = tokens // PAGE
    table = torch.ones(batch * pages, dtype=torch.int32, device=gu.DEV)
    q = torch.ones((batch * n, 1, D), dtype=torch.bfloat16, device=gu.DEV)
    out, lse = torch.full_like(q, float("nan")), torch.full((batch * n, 1), float("nan"), device=gu.DEV)
    ws = _ws(batch)
    kap.chunk_attn(q, gu.i32(np.arange(batch + 1) * n), pool, gu.i32(np.arange(batch + 1) * pages), table, gu.i32([tokens] * batch), out, ws, lse=lse)
    ws.check()
    assert bool((out.view(-1, D) == value).all())                 # weights of 1, whose sums are whole numbers: 2^24 is not passed without fresh sums
    seen = tokens - n + 1 + torch.arange(n, device=gu.DEV, dtype=torch.float64)
    assert float((lse.view(batch, n).double() - seen.log()).abs().max()) <= LSE


def _expected(q, pool, table, length, n, scale, window=0, sink=0):
    """rows of one sequence whose block table repeats few pages: (out, lse, weighted mean of |V|) in 64 bits; q [n, heads, D], one KV head"""
    kv = pool[:, :, 0].double()                                    # [pages, 2, PAGE, D]
    keys, values = kv[:, 0].reshape(-1, D), kv[:, 1].reshape(-1, D)
    z = torch.einsum("nhd,td->nht", q.double(), keys) * scale
    outs = []
    for j in range(n):
        p = length - n + j
        count = np.zeros((len(kv), PAGE), dtype=np.int64)
        spans = [(0, p + 1)] if not window or p - window < sink else [(0, sink), (p - window + 1, p + 1)]
        for lo, hi in spans:
            whole = table[-(-lo // PAGE):hi // PAGE]
            if -(-lo // PAGE) <= hi // PAGE:
                count += np.bincount(whole, minlength=len(kv))[:, None]
                if lo % PAGE:
                    count[table[lo // PAGE], lo % PAGE:] += 1
                if hi % PAGE:
                    count[table[hi // PAGE], :hi % PAGE] += 1
            else:
                count[table[lo // PAGE], lo % PAGE:hi % PAGE] += 1
        c = torch.from_numpy(count.reshape(-1)).to(gu.DEV).double()
        lse = torch.logsumexp(z[j] + c.log(), -1)
        w = torch.exp(z[j] - lse[:, None]) * c
        outs.append((w @ values, lse, w @ values.abs()))
    return [torch.stack(x) for x in zip(*outs)]


# (rows, context) of each sequence: units of one and of two tiles that a CTA does whole; cut ones on the tape; rows that all walk together, whole and in pieces
@pytest.mark.parametrize("sequences,heads,window,sink", [
    ([(1, 400_000 + 17 * b) for b in range(148)], 4, 0, 0),
    ([(70 + b % 80, 180_000 + 333 * b) for b in range(148)], 2, 0, 0),
    ([(1, 2 ** 25 + 5), (1, 2 ** 25 - 1000)], 8, 0, 0),
    ([(130, 2 ** 24 - 3), (200, 2 ** 24), (40, 2 ** 24)], 1, 0, 0),
    ([(150 * 256, 320_001)], 1, 0, 0),
    ([(300, 5_000_000)], 1, 0, 0),
    ([(300, 7_000_000)], 1, 5_000_000, 33),
])
def test_long_contexts(sequences, heads, window, sink):
    g = torch.Generator(device=gu.DEV).manual_seed(len(sequences))
    rng = np.random.default_rng(len(sequences))
    distinct, scale = 64, D ** -0.5
    pool = torch.randn((distinct, 2, 1, PAGE, D), device=gu.DEV, generator=g).mul_(0.5).to(torch.bfloat16)
    n_q, ctx = np.array(sequences).T
    lists = (ctx + PAGE - 1) // PAGE
    q_at, bt_at = (np.concatenate([[0], np.cumsum(x)]) for x in (n_q, lists))
    table = rng.integers(0, distinct, int(bt_at[-1])).astype(np.int32)
    q = torch.randn((int(q_at[-1]), heads, D), device=gu.DEV, generator=g).to(torch.bfloat16)
    out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device=gu.DEV)
    ws = _ws(len(n_q))
    args = q, gu.i32(q_at), pool, gu.i32(bt_at), gu.i32(table), gu.i32(ctx)
    kap.chunk_attn(*args, out, ws, lse=lse, window=window, n_sink=sink)
    ws.check()
    for b in {0, 1, len(n_q) // 2, len(n_q) - 1} & set(range(len(n_q))):
        for lo in {0, 5, int(n_q[b]) // 2, int(n_q[b]) - 2}:
            lo = max(lo, 0)
            hi = min(lo + 2, int(n_q[b]))
            if lo >= hi:
                continue
            rows = slice(int(q_at[b]) + lo, int(q_at[b]) + hi)
            o, l, size = _expected(q[rows], pool, table[bt_at[b]:bt_at[b + 1]], int(ctx[b] - n_q[b]) + hi, hi - lo, scale, window, sink)
            assert float((lse[rows].double() - l).abs().max()) <= LSE
            bound = 2.0 ** -8 * (size + o.abs()) + (SUM + 2e-4) * size
            assert bool(((out[rows].double() - o).abs() <= bound).all())
    again, lse_again = torch.empty_like(out), torch.empty_like(lse)
    kap.chunk_attn(*args, again, ws, lse=lse_again, window=window, n_sink=sink)
    ws.check()
    assert torch.equal(out, again) and torch.equal(lse, lse_again)


@pytest.mark.parametrize("n,heads", [(1, 4), (200, 1)])
def test_a_query_with_nan_behind_a_long_context(n, heads):
    distinct, batch, tokens = 8, 148, 400_000
    g = torch.Generator(device=gu.DEV).manual_seed(9)
    pool = torch.randn((distinct, 2, 1, PAGE, D), device=gu.DEV, generator=g).mul_(0.5).to(torch.bfloat16)
    pages = tokens // PAGE
    table = gu.i32(np.random.default_rng(9).integers(0, distinct, batch * pages))
    q = torch.randn((batch * n, heads, D), device=gu.DEV, generator=g).to(torch.bfloat16)
    ws = _ws(batch)
    results = []
    for bad in (False, True):
        if bad:
            q[n - 1, heads - 1, 3] = float("nan")
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=gu.DEV)
        kap.chunk_attn(q, gu.i32(np.arange(batch + 1) * n), pool, gu.i32(np.arange(batch + 1) * pages), table, gu.i32([tokens] * batch), out, ws, lse=lse)
        ws.check()
        results.append((out, lse))
    (out, lse), (bad_out, bad_lse) = results
    assert bool(bad_out[n - 1, heads - 1].isnan().all()) and bool(bad_lse[n - 1, heads - 1].isnan())
    bad_out[n - 1, heads - 1], bad_lse[n - 1, heads - 1] = out[n - 1, heads - 1], lse[n - 1, heads - 1]
    assert torch.equal(out, bad_out) and torch.equal(lse, bad_lse)
