"""kap_sample_tokens with NaN among its parameters: each one alone, in every combination of filters, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from test_gpu_sample import check, definition, f32, run, settings

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.mark.parametrize("filters", ["m", "tm", "km", "pm", "tkpm"])
@pytest.mark.parametrize("vocab", [40, 3001, 50257])
def test_a_nan_min_p_is_no_filter(vocab, filters):
    rng = np.random.default_rng(vocab)
    rows = 8
    x = f32(rng.normal(0, 2.5, (rows, vocab)))
    s = {n: v for n, v in settings(rng, rows).items() if n in filters}
    s["m"] = np.where(np.arange(rows) % 2 == 0, NAN, s["m"])
    u = rng.random(rows)
    got = check(x, u, **s)
    without = run(x, u, **{**s, "m": np.where(np.arange(rows) % 2 == 0, 0.0, s["m"])})
    np.testing.assert_array_equal(got, without[0])


@pytest.mark.parametrize("filters", ["", "t", "k", "p", "m", "tkpm"])
def test_a_nan_uniform_number_is_zero(filters):
    rng = np.random.default_rng(4)
    rows, vocab = 6, 5003
    x = rng.normal(0, 2.0, (rows, vocab))
    s = {n: v for n, v in settings(rng, rows).items() if n in filters}
    nan, zero = run(f32(x), [NAN] * rows, **s), run(f32(x), [0.0] * rows, **s)
    np.testing.assert_array_equal(nan[0], zero[0])
    np.testing.assert_array_equal(nan[1], zero[1])


def test_nan_temperature_is_greedy_and_nan_top_p_no_filter():
    rng = np.random.default_rng(5)
    x = rng.normal(0, 2.0, (4, 777)).astype(np.float32)
    token, logprob = run(f32(x), rng.random(4), t=[NAN] * 4, k=[5] * 4, p=[0.5] * 4, m=[NAN] * 4)
    np.testing.assert_array_equal(token, x.argmax(1))
    assert (logprob == 0).all()
    u = rng.random(4)
    got = run(f32(x), u, p=[NAN] * 4, m=[NAN] * 4)[0]
    want = [definition(x[r].astype(np.float64), float(np.float32(u[r])))[0] for r in range(4)]
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("rows", [3, 400])
def test_an_endless_temperature_draws_evenly(rows):
    # every weight is 1: token and log-probability follow from the counts alone, whichever way the rows go
    rng = np.random.default_rng(6)
    vocab = 9000
    x, u = f32(rng.normal(0, 3.0, (rows, vocab))), rng.random(rows)
    t = [np.inf] * rows
    for s, n in ((dict(), 9000), (dict(k=[700] * rows), 700), (dict(p=[0.25] * rows), 2250), (dict(k=[4000] * rows, p=[0.25] * rows), 1000), (dict(m=[0.5] * rows), 9000)):
        token, logprob = run(x, u, t=t, **s)
        assert (np.abs(logprob + np.log(n)) <= 2.0 ** -24 * np.log(n) + 1e-9).all()
        for r in range(3):
            kept = np.sort(np.argsort(-x[r].cpu().numpy(), kind="stable")[:n])
            assert token[r] == kept[int(np.float64(np.float32(u[r])) * n)]
