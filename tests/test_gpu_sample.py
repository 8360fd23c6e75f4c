"""kap_sample_tokens on the GPU against the definition in 64 bits on the host.

Tokens are compared exactly: both sides decide by sums in 64 bits, which differ by about 1e-13 of the total, and the seeds are
fixed.  The log-probability is a 64-bit value rounded to fp32 once: 2^-24 of it, plus 1e-9 for what the sums differ by."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap

pytestmark = pytest.mark.gpu
LOWEST = float(np.finfo(np.float32).min)


def definition(x, u, t=1.0, k=0, p=1.0, m=0.0):
    """one row, x float64; returns (token, logprob)"""
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == -np.inf:
        return -1, -np.inf
    if not t > 0:
        return int(np.argmax(x)), 0.0
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        z = np.where(x == top, 0.0, (x - top) / t)
        w = np.exp(z)
        order = np.lexsort((np.arange(x.size), -x))
        if 0 < k < x.size:
            order = order[:k]
        if p < 1:
            upto = np.cumsum(w[order])
            before = np.concatenate([[0.0], upto[:-1]])
            n = max(1, int((before < p * upto[-1]).sum()))
            order = order[:n]
        kept = np.zeros(x.size)
        kept[order] = w[order]
        if m > 0:
            kept[~(z >= np.log(m))] = 0.0
    upto = np.cumsum(kept)
    token = int(np.searchsorted(upto, u * upto[-1], side="right"))
    if token >= x.size:
        token = int(np.nonzero(kept)[0][-1])
    return token, z[token] - np.log(upto[-1])


def f32(a):
    return torch.from_numpy(np.asarray(a, dtype=np.float32)).to(gu.DEV)


def run(logits, u, t=None, k=None, p=None, m=None, stream=None):
    rows = logits.shape[0]
    token = torch.full((rows,), -7, dtype=torch.int32, device=gu.DEV)
    logprob = torch.full((rows,), float("nan"), device=gu.DEV)
    kap.sample_tokens(logits, f32(u), token, logprob, temperature=None if t is None else f32(t), top_k=None if k is None else gu.i32(k),
                      top_p=None if p is None else f32(p), min_p=None if m is None else f32(m), stream=stream)
    torch.cuda.synchronize()
    return token.cpu().numpy(), logprob.double().cpu().numpy()


def check(logits, u, t=None, k=None, p=None, m=None):
    got, lp = run(logits, u, t, k, p, m)
    x = logits.double().cpu().numpy()
    at = lambda a, r, off: off if a is None else np.float32(a[r]).astype(np.float64)   # noqa: E731
    for r in range(x.shape[0]):
        token, ref = definition(x[r], float(np.float32(u[r])), float(at(t, r, 1.0)), 0 if k is None else int(k[r]), float(at(p, r, 1.0)), float(at(m, r, 0.0)))
        assert got[r] == token, f"row {r}: token {got[r]}, expected {token} (logprob {lp[r]} / {ref})"
        assert lp[r] == ref or abs(lp[r] - ref) <= 2.0 ** -24 * abs(ref) + 1e-9, f"row {r}: logprob {lp[r]}, expected {ref}"
    return got


def settings(rng, rows):
    return dict(t=rng.uniform(0.3, 1.5, rows), k=rng.integers(1, 60, rows), p=rng.uniform(0.3, 0.99, rows), m=rng.uniform(0.0, 0.3, rows))


FILTERS = ["", "t", "tk", "tp", "tm", "tkp", "tpm", "kpm", "tkpm"]


@pytest.mark.parametrize("filters", FILTERS)
@pytest.mark.parametrize("vocab", [1, 2, 3, 31, 257, 4099, 50257, 128256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sizes_types_and_filters(vocab, filters, dtype):
    rng = np.random.default_rng(vocab * 16 + len(filters))
    rows = 9 if vocab < 50000 else 5
    x = rng.normal(0, 2.5, (rows, vocab))
    x[:, rng.integers(0, vocab, 12)] += rng.uniform(0, 9, 12)
    s = {n: v for n, v in settings(rng, rows).items() if n in filters}
    check(torch.from_numpy(x).to(gu.DEV).to(dtype), rng.random(rows), **s)


@pytest.mark.parametrize("filters", FILTERS)
@pytest.mark.parametrize("spread", [0.0, 1e-3, 0.3, 30.0, 3000.0])
def test_flat_and_peaked_rows(filters, spread):
    rng = np.random.default_rng(7)
    rows, vocab = 12, 20011
    x = rng.normal(0, 1, (rows, vocab)) * spread
    s = {n: v for n, v in settings(rng, rows).items() if n in filters}
    check(f32(x), rng.random(rows), **s)


@pytest.mark.parametrize("filters", ["tk", "tp", "tkp", "tkpm"])
@pytest.mark.parametrize("step", [0.5, 4.0])
def test_equal_logits_rank_by_index(filters, step):
    rng = np.random.default_rng(11)
    rows, vocab = 40, 3001
    x = np.round(rng.normal(0, 2, (rows, vocab)) / step) * step
    s = {n: v for n, v in settings(rng, rows).items() if n in filters}
    if "k" in s:
        s["k"] = rng.integers(1, vocab, rows)
    check(f32(x), rng.random(rows), **s)


@pytest.mark.parametrize("vocab", [2, 12, 30, 716, 2048, 40000])
@pytest.mark.parametrize("value", [0.0, -9984.0, np.inf, 1e-42])
def test_equal_logits_split_by_top_p_exactly(vocab, value):
    # n equal logits have n equal weights: p = 1/2, 1/4 and 3/4 of them end on a token when 4 divides n, and the next one stays out
    n = vocab // 4 * 4 if vocab > 2 else 2
    x = np.full((9, vocab), -np.inf)
    x[:, np.random.default_rng(vocab).permutation(vocab)[:n]] = value
    p = np.repeat([0.5, 0.25, 0.75], 3) if vocab > 2 else np.full(9, 0.5)
    got = check(f32(x), np.tile([0.0, 0.6, 1.0 - 2.0 ** -24], 3), t=np.tile([1.0, 0.3, 1e30], 3), p=p)
    at = np.nonzero(np.isfinite(x[0]) | (x[0] == np.inf))[0]
    assert (got[2::3] == at[(p[2::3] * n).astype(int) - 1]).all()


def test_ends_of_the_parameter_ranges():
    rng = np.random.default_rng(3)
    vocab = 1111
    ks = [-5, 0, 1, 2, vocab - 1, vocab, vocab + 1, 2 ** 31 - 1]
    ps = [-1.0, 0.0, 1e-30, 0.5, 1.0 - 2.0 ** -24, 1.0, 2.0, float("nan")]
    ms = [-1.0, 0.0, 1e-38, 0.5, 1.0, 1e-45, 0.999999, 0.1]
    ts = [0.0, -1.0, float("nan"), 1e-6, 1e-3, 1.0, 100.0, 1e30]
    us = [0.0, 2.0 ** -24, 0.25, 0.5, 0.75, 1.0 - 2.0 ** -24, 1.0 - 2.0 ** -23, 0.1]
    rows = 8
    x = rng.normal(0, 3, (rows, vocab))
    for a in range(8):
        roll = lambda v, n: np.roll(np.asarray(v, dtype=np.float64), n)               # noqa: E731
        check(f32(x), us, t=roll(ts, a), k=np.roll(np.array(ks, dtype=np.int64), 2 * a).astype(np.int32), p=roll(ps, 3 * a), m=roll(ms, 5 * a))
        check(f32(x), us, t=[0.9] * 8, k=np.roll(np.array(ks, dtype=np.int64), a).astype(np.int32))
        check(f32(x), us, t=[0.9] * 8, p=roll(ps, a))
        check(f32(x), us, t=[0.9] * 8, m=roll(ms, a))


@pytest.mark.parametrize("mask", [-np.inf, LOWEST, np.nan])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_rows(mask, dtype):
    rng = np.random.default_rng(5)
    rows, vocab = 12, 7003
    x = rng.normal(0, 2, (rows, vocab))
    for r in range(rows):
        x[r, rng.permutation(vocab)[:vocab - r]] = mask                              # r tokens left; row 0: none
    logits = torch.from_numpy(x).to(gu.DEV).to(dtype)
    for filters in FILTERS:
        s = {n: v for n, v in settings(rng, rows).items() if n in filters}
        check(logits, rng.random(rows), **s)
    check(logits, rng.random(rows), t=[0.0] * rows)


def test_infinite_logits():
    rng = np.random.default_rng(6)
    x = rng.normal(0, 2, (4, 999))
    x[0, [5, 800]] = np.inf
    x[1, 998] = np.inf
    x[2, [0, 1, 2]] = [np.inf, -np.inf, np.nan]
    x[3, 7] = 3.0e38
    for filters in FILTERS:
        s = {n: v for n, v in settings(rng, 4).items() if n in filters}
        for u in (0.0, 0.3, 0.9):
            check(f32(x), [u] * 4, **s)


def test_far_tokens_keep_their_small_weights():
    # u = 0 draws the first token of any weight, however small; weights below the smallest normal 64-bit number are none
    x = np.zeros((3, 300))
    x[0, :] = [-700.0] * 299 + [0.0]
    x[1, :] = [-1000.0] * 299 + [0.0]
    x[2, :] = [-30.0] * 299 + [0.0]
    token, _ = run(f32(x), [0.0, 0.0, 0.0])
    assert token.tolist() == [0, 299, 0]


@pytest.mark.parametrize("offset", [0, 1, 2, 3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_alignment(offset, dtype):
    rng = np.random.default_rng(8)
    rows, vocab = 6, 5003
    store = torch.full((rows, vocab + 9), 50.0, device=gu.DEV, dtype=dtype)           # what lies around a row must not be drawn
    view = store[:, offset:offset + vocab]
    view.copy_(torch.from_numpy(rng.normal(0, 2, (rows, vocab))))
    check(view, rng.random(rows), **settings(rng, rows))
    check(view[::2], rng.random(3))


@pytest.mark.parametrize("vocab", [200003, 262144])
def test_large_vocabularies(vocab):
    rng = np.random.default_rng(9)
    for spread in (0.5, 3.0):
        x = rng.normal(0, spread, (3, vocab))
        check(f32(x), rng.random(3))
        check(f32(x), rng.random(3), **settings(rng, 3))


@pytest.mark.parametrize("vocab,dtype", [(1, torch.float32), (5, torch.bfloat16), (129, torch.float32), (4099, torch.bfloat16), (50257, torch.float32),
                                         (128256, torch.float32), (128256, torch.bfloat16), (262144, torch.float32)])
def test_many_rows_without_filters(vocab, dtype):
    rng = np.random.default_rng(vocab)
    rows = 70 if vocab < 60000 else 52
    x = rng.normal(0, 1, (rows, vocab)) * rng.choice([0.0, 0.01, 1.0, 3.0, 50.0], (rows, 1))
    x[0, rng.integers(0, vocab, 3)] = np.inf
    x[1] = -np.inf
    x[2, rng.permutation(vocab)[:vocab - 1]] = np.nan
    x[3, rng.permutation(vocab)[:max(0, vocab - 40)]] = -np.inf
    x[4, rng.permutation(vocab)[:max(0, vocab - 7)]] = LOWEST
    t, u = rng.uniform(0.2, 2.0, rows), rng.random(rows)
    t[5:9] = [0.0, -1.0, 1e-6, 1e30]
    t[0] = 3e38 if vocab > 3 else 1.0
    x[12, ::2], t[12] = -0.0, 1e-37
    u[9:12] = [0.0, 1.0 - 2.0 ** -24, 2.0 ** -24]
    store = torch.full((rows, vocab + 9), 60.0, device=gu.DEV, dtype=dtype)
    for offset in (0, 1, 3):
        view = store[:, offset:offset + vocab]
        view.copy_(torch.from_numpy(x))
        check(view, u, t=t)
        store.fill_(60.0)
    # the same rows, few at a time, go another way and draw the same tokens
    logits = torch.from_numpy(x).to(gu.DEV).to(dtype)
    many = run(logits, u, t)
    for r0 in range(0, rows, 20):
        some = run(logits[r0:r0 + 20].contiguous(), u[r0:r0 + 20], t[r0:r0 + 20])
        np.testing.assert_array_equal(some[0], many[0][r0:r0 + 20])


def test_frequencies_follow_the_distribution():
    # 2^14 evenly spread numbers: every token comes within one of its share of them
    x = np.array([[0.0, 1.0, 2.0, -1.0, 0.5]])
    n = 1 << 14
    token, _ = run(f32(np.repeat(x, n, 0)), (np.arange(n) + 0.5) / n)
    share = np.exp(x[0]) / np.exp(x[0]).sum() * n
    assert (np.abs(np.bincount(token, minlength=5) - share) <= 1.0).all()


def test_rows_are_independent_and_runs_repeat():
    rng = np.random.default_rng(10)
    rows, vocab = 300, 30011
    x, u, s = f32(rng.normal(0, 2.5, (rows, vocab))), rng.random(rows), settings(rng, rows)
    first = run(x, u, **s)
    for _ in range(2):
        again = run(x, u, **s)
        np.testing.assert_array_equal(again[0], first[0])
        np.testing.assert_array_equal(again[1], first[1])
    pick = rng.permutation(rows)[:17]
    some = run(x[torch.from_numpy(pick).to(gu.DEV)].contiguous(), u[pick], **{n: v[pick] for n, v in s.items()})
    np.testing.assert_array_equal(some[0], first[0][pick])
    np.testing.assert_array_equal(some[1], first[1][pick])


def test_graph_capture_and_two_streams():
    rng = np.random.default_rng(12)
    rows, vocab = 7, 40009
    x = [f32(rng.normal(0, 2.5, (rows, vocab))) for _ in range(2)]
    u, t, k, p = f32(rng.random(rows)), f32([0.8] * rows), gu.i32([50] * rows), f32([0.9] * rows)
    want = [run(v, u.cpu().numpy(), t.cpu().numpy(), k.cpu().numpy(), p.cpu().numpy())[0] for v in x]
    work, token = x[0].clone(), [torch.zeros(rows, dtype=torch.int32, device=gu.DEV) for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kap.sample_tokens(work, u, token[0], temperature=t, top_k=k, top_p=p)
    for i in (1, 0, 1):
        work.copy_(x[i])
        graph.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(token[0].cpu().numpy(), want[i])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                kap.sample_tokens(x[i], u, token[i], temperature=t, top_k=k, top_p=p)
    torch.cuda.synchronize()
    for i in range(2):
        np.testing.assert_array_equal(token[i].cpu().numpy(), want[i])


def test_binding_refuses_what_it_cannot_pass_on():
    x = torch.zeros(4, 10, device=gu.DEV)
    u, token = torch.zeros(4, device=gu.DEV), torch.zeros(4, dtype=torch.int32, device=gu.DEV)
    for args, kw in (((x.half(), u, token), {}), ((x.t(), u, token), {}), ((x, u.double(), token), {}), ((x, u[:3], token), {}),
                     ((x, u, token.long()), {}), ((x, u, token), dict(top_k=u)), ((x, u, token), dict(temperature=token))):
        with pytest.raises(kap.KapError) as e:
            kap.sample_tokens(*args, **kw)
        assert e.value.code == kap.ERR_INVALID_ARG
