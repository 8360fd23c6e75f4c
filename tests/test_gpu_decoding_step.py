"""Decoding steps of a small two-layer model with the three calls together: kap_append_kv_rope places the new tokens,
kap_shared_prefix_attn reads them with the groups' shared pages, kap_sample_tokens draws the next token of every row.  Each stage is
held against its definition in 64 bits on what the stage before it left (tolerances: see the tests of the single calls), and a
captured step replayed over the same start must repeat the eager run bit for bit."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap
from test_gpu_append_rope import _rotated
from test_gpu_sample import definition
from test_gpu_shared_prefix import D, PAGE, Case

pytestmark = pytest.mark.gpu
VOCAB, WIDTH, LAYERS, STEPS = 1003, 256, 2, 6


class Decoder:
    def __init__(self, layout, groups, hq=8, hkv=2, dtype=torch.float32):
        self.hq, self.hkv, self.layout, self.dtype = hq, hkv, layout, dtype
        g = torch.Generator(device=gu.DEV).manual_seed(7)
        # a list has room for all steps; what lies behind the contexts is finite (the contexts grow over it)
        self.case = [Case(50 + i, groups, hq, hkv, layout, spare=2, poison=0.25) for i in range(LAYERS)]
        c = self.case[0]
        self.rows, self.batch = int(c.n_q.sum()), len(c.n_q)
        rand = lambda *s, by=1.0: torch.randn(s, device=gu.DEV, generator=g).mul_(by)     # noqa: E731
        self.embed = rand(VOCAB, WIDTH).to(torch.bfloat16)
        self.qkv = [rand(WIDTH, (hq + 2 * hkv) * D, by=WIDTH ** -0.5).to(torch.bfloat16) for _ in range(LAYERS)]
        self.back = [rand(hq * D, WIDTH, by=(hq * D) ** -0.5).to(torch.bfloat16) for _ in range(LAYERS)]
        self.head = rand(WIDTH, VOCAB, by=2 * WIDTH ** -0.5).to(torch.bfloat16)
        self.inv = (10000.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))).float().to(gu.DEV)
        self.u = torch.rand((STEPS, self.rows), device=gu.DEV, generator=g)
        rng = np.random.default_rng(3)
        self.t = rng.choice([0.0, 0.7, 1.0], self.rows).astype(np.float32)
        self.k = rng.choice([0, 1, 40], self.rows).astype(np.int32)
        self.p = rng.choice([0.5, 0.9, 1.0], self.rows).astype(np.float32)
        self.filters = dict(temperature=torch.from_numpy(self.t).to(gu.DEV), top_k=gu.i32(self.k), top_p=torch.from_numpy(self.p).to(gu.DEV))
        self.q_indptr = gu.i32(c.q_indptr)
        self.tables = [(gu.i32(x.bt_indptr), gu.i32(x.bt)) for x in self.case]
        self.start_pools = [x.pool.clone() for x in self.case]
        self.start = gu.i32(np.random.default_rng(4).integers(0, VOCAB, self.rows))
        self.ws = c.workspace()
        self.token = torch.empty(self.rows, dtype=torch.int32, device=gu.DEV)
        self.logprob = torch.empty(self.rows, device=gu.DEV)
        self.ctx = [torch.empty(self.batch, dtype=torch.int32, device=gu.DEV) for _ in range(LAYERS)]
        self.uniform = torch.empty(self.rows, device=gu.DEV)
        self.status = torch.zeros(1, dtype=torch.int32, device=gu.DEV)
        self.reset()

    def reset(self):
        for x, was, ctx in zip(self.case, self.start_pools, self.ctx):
            x.pool.copy_(was)
            ctx.copy_(gu.i32(x.ctx))
        self.token.copy_(self.start)

    def step(self, seen=None):
        """one step on the current stream; `seen` is called with what each stage left"""
        seen = seen or (lambda *a: None)
        stream = torch.cuda.current_stream()
        hidden = self.embed[self.token.long()]
        for i, x in enumerate(self.case):
            qkv = (hidden @ self.qkv[i]).view(self.rows, -1, D)
            q, k, v = qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hkv], qkv[:, self.hq + self.hkv:]
            q_out, out = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty(self.rows, self.hq, D, dtype=torch.bfloat16, device=gu.DEV)
            lse = torch.empty(self.rows, self.hq, device=gu.DEV)
            kap.append_kv_rope(q, k, v, x.pool, *self.tables[i], self.ctx[i], self.inv, q_out=q_out, new_indptr=self.q_indptr,
                               device_status=self.status, stream=stream, kv_layout=self.layout)
            seen("append", i, qkv, q_out)
            kap.shared_prefix_attn(q_out, self.q_indptr, x.pool, *self.tables[i], self.ctx[i], out, self.ws, lse=lse, stream=stream)
            seen("attend", i, q_out, out, lse)
            hidden = hidden + out.view(self.rows, -1) @ self.back[i]
        logits = (hidden @ self.head).to(self.dtype)
        kap.sample_tokens(logits, self.uniform, self.token, self.logprob, stream=stream, **self.filters)
        seen("sample", logits)

    def run(self, one):
        history = []
        for s in range(STEPS):
            self.uniform.copy_(self.u[s])
            one()
            torch.cuda.synchronize()
            history.append((self.token.cpu().numpy().copy(), self.logprob.cpu().numpy().copy()))
        self.ws.check()
        assert int(self.status.item()) == 0
        return history

    # ---- the definitions
    def check_stage(self, what, *a):
        torch.cuda.synchronize()
        getattr(self, "check_" + what)(*a)

    def check_append(self, i, qkv, q_out):
        x, ctx = self.case[i], self.ctx[i].cpu().numpy()
        pos = np.concatenate([L - n + np.arange(n) for L, n in zip(ctx, x.n_q)])
        seq = np.repeat(np.arange(self.batch), x.n_q)
        angle = pos[:, None] * self.inv.double().cpu().numpy()
        rows = qkv.double().cpu().numpy()
        pages = torch.from_numpy(x.bt[x.bt_indptr[seq] + pos // PAGE].astype(np.int64)).to(gu.DEV)
        slots = torch.from_numpy(pos % PAGE).to(gu.DEV)
        heads = x.heads_first()
        for got, h0, h1 in ((q_out, 0, self.hq), (heads[pages, 0, :, slots], self.hq, self.hq + self.hkv)):
            ref, size = _rotated(rows[:, h0:h1], angle, D, False)
            assert (np.abs(got.double().cpu().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -20 * size).all()
        assert torch.equal(heads[pages, 1, :, slots], qkv[:, self.hq + self.hkv:])

    def check_attend(self, i, q, out, lse):
        x, ctx = self.case[i], self.ctx[i].cpu().numpy()
        x.q, x.call = q, lambda *a: (out, lse)
        x.check(ctx)

    def check_sample(self, logits):
        x, token, lp = logits.double().cpu().numpy(), self.token.cpu().numpy(), self.logprob.double().cpu().numpy()
        for r in range(self.rows):
            want, ref = definition(x[r], float(self.uniform[r]), float(self.t[r]), int(self.k[r]), float(self.p[r]))
            assert token[r] == want and abs(lp[r] - ref) <= 2.0 ** -24 * abs(ref) + 1e-9


GROUPS = [(9, [(1, 5), (4, 20), (1, 1), (2, 30)]), (0, [(3, 77)]), (70, [(1, 33)] * 40)]


@pytest.mark.parametrize("layout,dtype", [(kap.KV_HND, torch.float32), (kap.KV_NHD, torch.bfloat16)])
def test_steps_against_the_definitions_and_captured(layout, dtype):
    d = Decoder(layout, GROUPS, dtype=dtype)
    eager = d.run(lambda: d.step(d.check_stage))
    pools, ctx = [x.pool.clone() for x in d.case], [c.clone() for c in d.ctx]
    assert all((c.cpu().numpy() == x.ctx + STEPS * x.n_q).all() for c, x in zip(d.ctx, d.case))

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        d.reset()
        d.uniform.copy_(d.u[0])
        d.step()                                                               # library handles and workspaces before the capture
        d.reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        d.step()
    for _ in range(2):
        d.reset()
        for (token, lp), (want, want_lp) in zip(d.run(graph.replay), eager):
            np.testing.assert_array_equal(token, want)
            np.testing.assert_array_equal(lp, want_lp)
        assert all(torch.equal(x.pool, p) for x, p in zip(d.case, pools)) and all(torch.equal(a, b) for a, b in zip(d.ctx, ctx))


def test_steps_without_shared_pages_match_the_verification_call():
    d = Decoder(kap.KV_HND, [(0, [(4, 60)]), (0, [(4, 200)]), (0, [(4, 33)])])
    got = {}
    d.uniform.copy_(d.u[0])
    d.step(lambda what, *a: got.setdefault(what, [t.clone() if torch.is_tensor(t) else t for t in a]))
    i, q, out, lse = got["attend"]
    x = d.case[i]
    ws = kap.Workspace(max_rows_per_item=64, max_batch=d.batch)
    ws.schedule(x.lists, x.n_q, d.hq, d.hkv)
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    kap.verify_attn(q, d.q_indptr, x.pool, *d.tables[i], d.ctx[i], out2, ws, lse=lse2)
    ws.check()
    # each is within 2^-8 of its weights and 2^-8 of its result of the definition
    size = x.pool[:, 1].float().abs().max().item()
    assert (out.double() - out2.double()).abs().max().item() <= 2 * (2.0 ** -8 + 1e-4 + 2.0 ** -8) * size
    # kap_verify_attn's small-row kernel sums the weights after their rounding to bf16: every term, and so the sum, is within 2^-8 of itself, and
    # the sum's logarithm within -ln(1 - 2^-8) < 2^-8 + 2^-16; the scores' errors add 2e-5 on either side
    assert (lse - lse2).abs().max().item() <= 2.0 ** -8 + 2.0 ** -16 + 4e-5


@pytest.mark.parametrize("layout", [kap.KV_HND, kap.KV_NHD])
def test_offsets_past_32_bits(layout):
    # the pages at the end of a pool of 4.6 G elements, and logits rows 2.2 G elements apart, give what the same data does at the front
    c = Case(77, [(6, [(1, 40), (2, 9)]), (40, [(2, 50)] * 20)], 32, 8, layout, spare=1, poison=0.0)
    n, pages = c.pool.shape[0], 140000
    first = pages - n
    far = torch.empty((pages,) + tuple(c.pool.shape[1:]), dtype=torch.bfloat16, device=gu.DEV)
    far[first:] = c.pool
    table = gu.i32(c.bt), gu.i32(c.bt + first)
    rows, qi, bti, inv = int(c.n_q.sum()), gu.i32(c.q_indptr), gu.i32(c.bt_indptr), torch.full((64,), 0.01, device=gu.DEV)
    k, v = (torch.randn(rows, 8, D, device=gu.DEV).to(torch.bfloat16) for _ in range(2))
    ws, got = c.workspace(), []
    for pool, bt in zip((c.pool, far), table):
        ctx, out, q = gu.i32(c.ctx), torch.empty_like(c.q), torch.empty_like(c.q)
        status = torch.zeros(1, dtype=torch.int32, device=gu.DEV)
        kap.append_kv_rope(c.q, k, v, pool, bti, bt, ctx, inv, q_out=q, new_indptr=qi, device_status=status, kv_layout=layout)
        kap.shared_prefix_attn(q, qi, pool, bti, bt, ctx, out, ws)
        ws.check()
        assert int(status.item()) == 0
        got.append(out)
    assert torch.equal(*got) and torch.equal(far[first:], c.pool) and torch.isfinite(got[0].float()).all()
    del far
    stride, vocab = 2_200_000_003, 50257
    store = torch.empty(stride + vocab, dtype=torch.bfloat16, device=gu.DEV)
    logits = store.as_strided((2, vocab), (stride, 1))
    logits.copy_(torch.randn(2, vocab, device=gu.DEV))
    u, near, lp = torch.tensor([0.3, 0.8], device=gu.DEV), logits.contiguous(), torch.empty(2, device=gu.DEV)
    for filters in ({}, dict(top_p=torch.full((2,), 0.9, device=gu.DEV))):
        a, b = (torch.empty(2, dtype=torch.int32, device=gu.DEV) for _ in range(2))
        kap.sample_tokens(logits, u, a, lp, **filters)
        kap.sample_tokens(near, u, b, lp, **filters)
        assert torch.equal(a, b) and (a >= 0).all()
