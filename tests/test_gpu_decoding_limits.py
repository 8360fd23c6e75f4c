"""The decoding calls at the largest sizes that they take, and in uses next to the ordinary ones: other streams, the same call captured
several times, arrays longer than needed.  Tolerances as in the calls' own test files."""
import numpy as np
import pytest
import torch

import gpu_util as gu
import test_gpu_append_rope as append
import test_gpu_sample as sampling
from paper_2607_24260_b200 import kap
from test_gpu_shared_prefix import Case

pytestmark = pytest.mark.gpu
MOST = 16 * 512 * 99


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [MOST, MOST - 1, 16 * 512 * 97 + 1])
def test_the_largest_vocabularies(vocab, dtype):
    rng = np.random.default_rng(vocab)
    x = torch.from_numpy(rng.normal(0, 1.5, (2, vocab)).astype(np.float32)).to(gu.DEV).to(dtype)
    sampling.check(x, rng.random(2))
    sampling.check(x, rng.random(2), t=[0.0, 0.0])
    sampling.check(x, rng.random(2), p=[0.9, 0.5])
    sampling.check(x, rng.random(2), **sampling.settings(rng, 2))
    store = torch.zeros((2, vocab + 5), device=gu.DEV, dtype=dtype)
    store[:, 3:vocab + 3] = x
    sampling.check(store[:, 3:vocab + 3], rng.random(2), k=[700, 5], p=[0.99, 0.7])


def test_more_rows_than_clusters_fit_the_device():
    # 1500 rows with all filters: the grid runs in many waves, and equal rows get equal tokens
    rng = np.random.default_rng(1)
    x = sampling.f32(rng.normal(0, 2.5, (15, 20011))).repeat(100, 1)
    s = {n: np.tile(v, 100) for n, v in sampling.settings(rng, 15).items()}
    u = np.tile(rng.random(15), 100)
    token, logprob = sampling.run(x, u, **s)
    sampling.check(x[:15], u[:15], **{n: v[:15] for n, v in s.items()})
    assert (token.reshape(100, 15) == token[:15]).all() and (logprob.reshape(100, 15) == logprob[:15]).all()


@pytest.mark.parametrize("batch", [33, 1025, 3000])
def test_append_for_many_sequences(batch):
    rng = np.random.default_rng(batch)
    c = append.Case.__new__(append.Case)                                         # (its constructor has 64 pages at most; here each sequence has one)
    c.n_new, c.ctx = rng.integers(0, 3, batch), rng.integers(0, 14, batch)
    c.n_new[-1] = 2
    c.hq, c.hkv, c.rot, c.inter, c.layout, c.rows = 2, 1, 128, False, kap.KV_HND, int(c.n_new.sum())
    c.inv = (10000.0 ** (-np.arange(64) / 64)).astype(np.float32)
    c.bt_indptr, c.bt = np.arange(batch + 1, dtype=np.int32), rng.permutation(batch).astype(np.int32)
    c.qkv, c.pool = append.synth.normal_bf16((c.rows, 4, 128), 1.0, rng), append.synth.normal_bf16((batch, 2, 1, 16, 128), 0.5, rng)
    dev = gu.bits_to_dev(c.qkv)
    c.q, c.k, c.v = dev[:, :2], dev[:, 2:3], dev[:, 3:]
    c.d_pool, c.d_ctx, c.d_bt = gu.bits_to_dev(c.pool), gu.i32(c.ctx), (gu.i32(c.bt_indptr), gu.i32(c.bt))
    c.d_indptr, c.status = gu.i32(np.concatenate([[0], np.cumsum(c.n_new)])), torch.zeros(1, dtype=torch.int32, device=gu.DEV)
    c.check(c.call())


def test_append_captured_with_and_without_windows():
    # one graph with three steps of a batch: two windows of several tokens, then one token each; ctx_len moves on the device
    rng = np.random.default_rng(61)
    windows = [np.array([3, 0, 5]), np.array([1, 2, 0]), np.array([1, 1, 1])]
    ctx = np.array([13, 40, 0])
    steps, at = [], ctx.copy()
    for i, n in enumerate(windows):
        steps.append((n, at.copy(), gu.bits_to_dev(append.synth.normal_bf16((int(n.sum()), 4, 128), 1.0, rng))))
        at = at + n
    pages = (at + 15) // 16
    indptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
    table = rng.permutation(int(pages.sum())).astype(np.int32)
    start = gu.bits_to_dev(append.synth.normal_bf16((int(pages.sum()), 2, 1, 16, 128), 0.5, rng))
    inv = torch.from_numpy((10000.0 ** (-np.arange(64) / 64)).astype(np.float32)).to(gu.DEV)

    def run(pool, ctx_len, outs):
        for i, (n, _, qkv) in enumerate(steps):
            kap.append_kv_rope(qkv[:, :2], qkv[:, 2:3], qkv[:, 3:], pool, gu_indptr, gu_table, ctx_len, inv, outs[i], new_indptr=indptrs[i])

    gu_indptr, gu_table = gu.i32(indptr), gu.i32(table)
    indptrs = [None if i == 2 else gu.i32(np.concatenate([[0], np.cumsum(n)])) for i, (n, _, _) in enumerate(steps)]
    outs = [torch.zeros((qkv.shape[0], 2, 128), dtype=torch.bfloat16, device=gu.DEV) for _, _, qkv in steps]
    want_pool, want_ctx = start.clone(), gu.i32(ctx)
    run(want_pool, want_ctx, outs)
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    pool, ctx_len = start.clone(), gu.i32(ctx)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(pool, ctx_len, outs)
    for _ in range(3):
        pool.copy_(start)
        ctx_len.copy_(gu.i32(ctx))
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(pool, want_pool) and torch.equal(ctx_len, want_ctx) and all(torch.equal(a, b) for a, b in zip(outs, want))
    assert ctx_len.tolist() == at.tolist()


def test_calls_on_a_given_stream_follow_its_order():
    stream = torch.cuda.Stream()
    c = Case(62, [(40, [(1, 30)] * 40), (2, [(4, 60)])], poison=0.0)
    want = c.call()
    q, qi, pool, bti, btp, ctx = c.arrays()
    q2, out = torch.zeros_like(q), torch.zeros_like(q)
    torch.cuda.synchronize()
    for _ in range(10):
        with torch.cuda.stream(stream):
            out.zero_()
            q2.copy_(q)
        kap.shared_prefix_attn(q2, qi, pool, bti, btp, ctx, out, c.ws, stream=stream, sm_scale=c.scale)
        with torch.cuda.stream(stream):
            got = out.clone()
            q2.zero_()
        stream.synchronize()
        assert torch.equal(got, want[0])


def test_a_batch_of_many_sequences():
    rng = np.random.default_rng(63)
    Case(63, [(9, [(1, int(t)) for t in rng.integers(1, 60, 1200)]), (0, [(1, 5)] * 100)], 4, 1).check()
