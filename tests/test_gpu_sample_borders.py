"""kap_sample_tokens where the top-p border lies next to wide gaps between the values, against the definition in 64 bits.

The rows have more candidates at each value than one CTA finishes alone, and top_p is a given distance past the place where the
weight of a value is used up, so that the prefix reaches into the next one (or just not).  Exact tokens and log-probabilities as
everywhere (test_gpu_sample.py has the tolerances): a shortest prefix that is wrong by one token moves the log-probability by
1 / 10^4 here, and p times the whole lies 10^-6 of it or more from every border, far outside the 10^-13 by which sums differ."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from test_gpu_sample import check, definition, f32, run

pytestmark = pytest.mark.gpu


def row(rng, values, counts, vocab=None):
    x = np.repeat(np.asarray(values, dtype=np.float64), counts)
    if vocab is not None:
        x = np.concatenate([x, np.full(vocab - x.size, -np.inf)])
    return x[rng.permutation(x.size)]


def borders(values, counts, t, k=0):
    """the shares of the whole at which the weight of each value but the last is used up; with top-k of what that left"""
    z = np.asarray(values, dtype=np.float64) / t
    n = np.asarray(counts, dtype=np.int64)
    if k > 0:
        n = np.minimum(n, np.maximum(0, k - np.concatenate([[0], np.cumsum(n)[:-1]])))
    w = np.cumsum(n * np.exp(z - z[0]))
    return w[:-1] / w[-1]


LEVELS = [([3.0, 1.0, -1.0], [1, 1000, 4000]), ([2.0, -2.0], [600, 5000]), ([0.5, 0.0, -0.5], [700, 900, 3000]), ([1.5, -1e-30, -1.5], [600, 600, 4000]),
          ([1.0, 1.0 - 2.0 ** -8, -1.0], [600, 600, 3000]), ([-0.25, -1.25, -2.25], [513, 1000, 5000]), ([4.0, 1e-38, -1e-38], [3, 3000, 3000])]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("values,counts", LEVELS)
def test_top_p_just_past_a_gap(values, counts, dtype):
    rng = np.random.default_rng(len(counts) + counts[0])
    x, ps, ts = [], [], []
    for t in (1.0, 0.7):
        for b in borders(values, counts, t):
            for past in (-1e-4, -1e-5, 1e-5, 1e-4, 3e-4, 1e-3, 1e-2):
                if 0 < b * (1 + past) < 1:
                    x.append(row(rng, values, counts))
                    ps.append(b * (1 + past))
                    ts.append(t)
    logits = torch.from_numpy(np.stack(x)).to(gu.DEV).to(dtype)
    check(logits, rng.random(len(ps)), t=ts, p=ps)
    check(logits, np.full(len(ps), 1.0 - 2.0 ** -24), t=ts, p=ps)


@pytest.mark.parametrize("values,counts", LEVELS[:4])
def test_top_p_just_past_a_gap_of_what_top_k_left(values, counts):
    rng = np.random.default_rng(counts[0])
    x, ps, ks = [], [], []
    for k in (sum(counts) - 1500, sum(counts[:-1]) + 700, sum(counts) - 1):
        for b in borders(values, counts, 1.0, k):
            for past in (-1e-4, 1e-5, 1e-4, 1e-3, 1e-2):
                if 0 < b * (1 + past) < 1:
                    x.append(row(rng, values, counts))
                    ps.append(b * (1 + past))
                    ks.append(k)
    check(f32(np.stack(x)), rng.random(len(ps)), k=ks, p=ps)


def test_rows_of_two_values():
    # values, counts and shares at random: every border may lie at the end of the first value, across zero or far from it
    rng = np.random.default_rng(21)
    rows, vocab = 600, 6000
    x, ps = [], []
    for _ in range(rows):
        first = int(rng.integers(513, 3000))
        values = np.sort(rng.normal(0, 1.5, 2))[::-1].astype(np.float32)
        counts = [first, vocab - first]
        x.append(row(rng, values, counts))
        b = borders(values, counts, 1.0)[0]
        ps.append(min(b * (1.0 + 10.0 ** rng.uniform(-5, -2)), 1 - 1e-6))
    check(f32(np.stack(x)), rng.random(rows), p=ps)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_weights_that_halve(dtype):
    # one value after another with half the weight: what is missing to p of the whole is always about what the next value weighs
    rng = np.random.default_rng(22)
    x, ps = [], []
    steps = np.arange(60)
    for first in (600, 900):
        values = np.round((8.0 - steps * np.log(2.0)) * 16) / 16
        counts = [first] + [40 + int(c) for c in rng.integers(0, 30, 59)]
        for share in np.concatenate([borders(values, counts, 1.0)[[0, 1, 5, 10, 20]] * (1 + 2e-6), [0.3, 0.9, 0.999, 0.9999, 1 - 1e-6]]):
            if share < 1:
                x.append(row(rng, values, counts, 6000))
                ps.append(share)
    check(torch.from_numpy(np.stack(x)).to(gu.DEV).to(dtype), rng.random(len(ps)), p=ps)


def test_large_vocabularies_with_gaps():
    rng = np.random.default_rng(23)
    x, ps = [], []
    for values, counts in (([3.0, 1.0, -1.0], [1, 30000, 98255]), ([1e-3, -1e-3], [28256, 100000]), ([40.0, -40.0], [600, 127656])):
        for past in (1e-5, 1e-3):
            for b in borders(values, counts, 1.0):
                x.append(row(rng, values, counts))
                ps.append(min(b * (1 + past), 1 - 1e-6))
    check(f32(np.stack(x)), rng.random(len(ps)), p=ps)


def test_the_definition_of_a_known_row():
    # one logit at 3, 1000 at 1 and 4000 at -1, p just past the second value's end: 1002 to 1009 tokens stay
    x = np.concatenate([[3.0], np.full(1000, 1.0), np.full(4000, -1.0)])
    w = np.exp(x - 3.0)
    for p in (0.6505, 0.6506, 0.651, 0.6511):
        upto = np.cumsum(w)
        kept = 1 + int((upto < float(np.float32(p)) * upto[-1]).sum())
        assert 1002 <= kept <= 1012
        token, logprob = definition(x, 1.0 - 2.0 ** -24, p=float(np.float32(p)))
        assert token == kept - 1
        check(f32(x[None]), [1.0 - 2.0 ** -24], p=[p])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_rows_beside_gaps_get_equal_tokens(dtype):
    # every row 150 times: whichever way its CTAs come through the search, the result is one
    rng = np.random.default_rng(24)
    x, ps = [], []
    for _ in range(20):
        values = np.sort(rng.normal(0, 2.0, int(rng.integers(2, 6))))[::-1]
        x.append(rng.choice(values, 17000))
        v, n = np.unique(x[-1], return_counts=True)
        share = rng.choice(np.cumsum(n[::-1] * np.exp(v[::-1] - v[-1]))[:-1]) / (n * np.exp(v - v[-1])).sum()
        ps.append(min(share * (1 + 10.0 ** rng.uniform(-6, -2)), 1 - 1e-6))
    x.append(np.sign(rng.normal(0, 1, 17000)) * 10.0 ** rng.uniform(-38, 1, 17000))
    ps.append(0.9999)
    copies, u = 150, rng.random(len(ps))
    logits = torch.from_numpy(np.stack(x)).to(gu.DEV).to(dtype)
    check(logits, u, p=ps)
    token, logprob = run(logits.repeat(copies, 1), np.tile(u, copies), p=np.tile(ps, copies))
    token, logprob = token.reshape(copies, -1), logprob.reshape(copies, -1)
    assert (token == token[0]).all() and (logprob == logprob[0]).all()


def test_rows_of_every_kind_and_shares_next_to_their_borders():
    rng = np.random.default_rng(25)
    for _ in range(40):
        rows, vocab = 24, int(np.exp(rng.uniform(np.log(600), np.log(20000))))
        x, p, t = np.empty((rows, vocab), dtype=np.float32), rng.uniform(0, 1, rows), 10.0 ** rng.uniform(-1.5, 1.5, rows)
        for r in range(rows):
            scale = 10.0 ** rng.uniform(-3, 2)
            x[r] = [lambda: rng.normal(0, scale, vocab), lambda: rng.choice(rng.normal(0, scale, 3), vocab),
                    lambda: np.round(rng.normal(0, 4, vocab)) * scale / 4, lambda: np.sign(rng.normal(0, 1, vocab)) * 10.0 ** rng.uniform(-38, 2, vocab),
                    lambda: rng.normal(0, 1e-3 * scale, vocab) + rng.choice([-3.0, 0.0, 3.0], vocab, p=[0.6, 0.3, 0.1]),
                    lambda: -np.log(2) * np.floor(rng.uniform(0, 40, vocab)) * scale][r % 6]()
            z = np.sort(x[r].astype(np.float64))[::-1]
            border = np.nonzero(np.diff(z) < 0)[0][:8]
            if border.size and r % 4:
                w = np.cumsum(np.exp((z - z[0]) / np.float64(np.float32(t[r]))))
                p[r] = min(w[rng.choice(border)] / w[-1] * (1 + 10.0 ** rng.uniform(-6, -2)), 1 - 1e-7)
        s = dict(t=t, p=p)
        if rng.random() < 0.3:
            s["k"] = rng.integers(1, vocab, rows)
        if rng.random() < 0.3:
            s["m"] = 10.0 ** rng.uniform(-6, 0, rows)
        check(f32(x), np.where(rng.random(rows) < 0.3, 1 - 2.0 ** -24, rng.random(rows)), **s)
