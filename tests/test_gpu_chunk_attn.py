"""kap_chunk_attn on the GPU against plain attention in 64 bits.

Tolerance of a result, as for the shared-prefix attention: each weight is rounded to bf16 for the product with V (at most 2^-8 of it), so
the weighted mean moves by at most 2^-8 of the weighted mean of |V|; a score is a fp32 sum of 128 products, off by less than
128 2^-23 sum |q k| scale (below 1e-4 for q ~ N(0, 1), k ~ N(0, 1/4) and scale 128^-1/2, whose sum |q k| scale stays below 6), which moves a
weight by as much of itself; the result is rounded to bf16 once (2^-8 of it).  lse: the same 1e-4 bounds its absolute error; the
typical one is 1e-6, and 2e-5 is asked for (an average over the row's scores).  With scores `hot` times as large all of these grow by `hot`."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap

pytestmark = pytest.mark.gpu
D, PAGE = 128, 16
HND, NHD = kap.KV_HND, kap.KV_NHD


class Case:
    """sequences: a list of (n_q, ctx_len); `before` and `behind` rows of q belong to nobody"""

    def __init__(self, seed, sequences, hq=8, hkv=2, layout=HND, window=0, sink=0, before=0, behind=3, scale=None, hot=1.0, pages=None):
        g = torch.Generator(device=gu.DEV).manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.hq, self.hkv, self.layout, self.window, self.sink, self.hot = hq, hkv, layout, window, sink, hot
        self.scale = D ** -0.5 if scale is None else scale
        self.n_q = np.array([n for n, _ in sequences], dtype=np.int64)
        self.ctx = np.array([c for _, c in sequences], dtype=np.int64)
        lists = (self.ctx + PAGE - 1) // PAGE
        self.bt_indptr = np.concatenate([[0], np.cumsum(lists)]).astype(np.int32)
        self.q_indptr = (before + np.concatenate([[0], np.cumsum(self.n_q)])).astype(np.int32)
        self.rows = int(self.q_indptr[-1]) + behind
        seen = [self.seen_pages(b) for b in range(len(self.n_q))]
        need = sum(len(x) for x in seen)
        self.n_pages = max(need + 2, pages or 0)
        # pages that no row sees: entries that are no pages at all
        self.bt = rng.choice(np.array([-1, self.n_pages, 2 ** 30], dtype=np.int32), int(lists.sum()))
        fresh = rng.permutation(self.n_pages)[:need] if pages is None else self.n_pages - 1 - np.arange(need)
        at = 0
        for b, x in enumerate(seen):
            self.bt[self.bt_indptr[b] + x] = fresh[at:at + len(x)]
            at += len(x)
        shape = (self.n_pages, 2, hkv, PAGE, D) if layout == HND else (self.n_pages, 2, PAGE, hkv, D)
        self.pool = torch.empty(shape, dtype=torch.bfloat16, device=gu.DEV).fill_(float("nan"))
        heads = self.heads_first()
        for b, x in enumerate(seen):                              # everything behind the contexts stays NaN
            for lo in range(0, len(x), 4096):
                part = x[lo:lo + 4096]
                new = (torch.randn((len(part), 2, hkv, PAGE, D), device=gu.DEV, generator=g) * (0.5 * hot)).to(torch.bfloat16)
                new[:, 1] /= hot
                token = torch.from_numpy(part[:, None] * PAGE + np.arange(PAGE)).to(gu.DEV)
                new = torch.where((token < int(self.ctx[b]))[:, None, None, :, None], new, float("nan"))
                heads[torch.from_numpy(self.bt[self.bt_indptr[b] + part].astype(np.int64)).to(gu.DEV)] = new
        self.q = torch.randn((self.rows, hq, D), device=gu.DEV, generator=g).to(torch.bfloat16)
        self.ws = None

    def heads_first(self):
        return self.pool if self.layout == HND else self.pool.transpose(2, 3)

    def seen_pages(self, b):
        page = np.arange((self.ctx[b] + PAGE - 1) // PAGE)
        if not self.n_q[b]:
            return page[:0]
        if not self.window:
            return page
        first = max(0, self.ctx[b] - self.n_q[b] - self.window + 1)
        return page[(page * PAGE + PAGE > first) | (page * PAGE < self.sink)]

    def workspace(self):
        ws = kap.Workspace(max_items=kap.chunk_attn_items(max_rows_per_item=64), max_rows_per_item=64, max_batch=max(1, len(self.n_q)))
        ws.set_kv_layout(self.layout)
        return ws

    def call(self, ws=None, stream=None, check=True):
        self.ws = ws or self.ws or self.workspace()
        out = torch.full_like(self.q, float("nan"))
        lse = torch.full(self.q.shape[:2], float("nan"), device=gu.DEV)
        kap.chunk_attn(self.q, gu.i32(self.q_indptr), self.pool, gu.i32(self.bt_indptr), gu.i32(self.bt), gu.i32(self.ctx), out, self.ws, lse=lse,
                       window=self.window, n_sink=self.sink, sm_scale=self.scale, stream=stream)
        if check:
            self.ws.check()
        return out, lse

    def expected(self, b, lo=0, hi=None):
        """out, lse and the weighted mean of |V| of rows lo .. hi - 1 of sequence b in 64 bits"""
        G = self.hq // self.hkv
        hi = int(self.n_q[b]) if hi is None else hi
        n, length, first = hi - lo, int(self.ctx[b]) - int(self.n_q[b]) + hi, int(self.q_indptr[b]) + lo
        t = torch.arange(max(length, 0), device=gu.DEV)
        if self.window:
            t = t[(t < self.sink) | (t > length - n - self.window)]
        p = torch.arange(length - n, length, device=gu.DEV)
        sees = t[None] <= p[:, None]
        if self.window:
            sees &= (t[None] > p[:, None] - self.window) | (t[None] < self.sink)
        entry = torch.from_numpy(self.bt[self.bt_indptr[b]:self.bt_indptr[b + 1]].astype(np.int64)).to(gu.DEV)
        kv = self.heads_first()[entry[t // PAGE], :, :, t % PAGE].double()          # [tokens, 2, Hkv, D]
        q = self.q[first:first + n].double().view(n, self.hkv, G, D)
        z = torch.einsum("nhgd,thd->hgnt", q, kv[:, 0]) * self.scale
        z = torch.where(sees, z, -torch.inf)
        lse = torch.logsumexp(z, -1)
        w = torch.exp(z - torch.where(lse == -torch.inf, 0.0, lse)[..., None])
        flat = lambda x: x.permute(2, 0, 1, *range(3, x.dim())).reshape(n, self.hq, *x.shape[3:])     # noqa: E731
        return [flat(x) for x in (torch.einsum("hgnt,thd->hgnd", w, kv[:, 1]), lse, torch.einsum("hgnt,thd->hgnd", w, kv[:, 1].abs()))]

    def check(self, out, lse, only=None, rows=None):
        """rows: so many rows at a time, the first, the last and some between"""
        parts = []
        for b in range(len(self.n_q)) if only is None else only:
            n = int(self.n_q[b])
            starts = [0] if rows is None or n <= rows else [0, n - rows] + list(range(rows, n - rows, max(rows, n // 5)))
            parts += [(b, lo, min(n, lo + (rows or n))) for lo in starts if n]
        for b, lo, hi in parts:
            first = int(self.q_indptr[b])
            rows = slice(first + lo, first + hi)
            o, l, size = self.expected(b, lo, hi)
            bound = 2.0 ** -8 * (size + o.abs()) + 2e-4 * self.hot * size + 1e-30
            err = (out[rows].double() - o).abs()
            assert bool((err <= bound).all()), f"sequence {b}: {int((err > bound).sum())} values off, worst {float((err / bound).max())} of the bound"
            assert bool(((lse[rows].double() - l).abs() <= 2e-5 * self.hot).masked_fill(l == -torch.inf, True).all()), f"sequence {b}: lse"
            assert torch.equal(lse[rows] == -torch.inf, l == -torch.inf)
        free = torch.ones(self.rows, dtype=torch.bool, device=gu.DEV)
        free[int(self.q_indptr[0]):int(self.q_indptr[-1])] = False
        assert bool(out[free].isnan().all()) and bool(lse[free].isnan().all()), "rows of nobody were written"


MIXED = [(1, 1), (300, 700), (1, 4097), (0, 50), (65, 65), (17, 33), (1, 16), (128, 1000), (0, 0), (1, 2000)]


@pytest.mark.parametrize("layout", [HND, NHD])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (2, 2), (1, 1), (6, 3), (16, 2), (32, 2)])
def test_mixed_batches(hq, hkv, layout):
    c = Case(1, MIXED, hq, hkv, layout, before=2)
    c.check(*c.call())


@pytest.mark.parametrize("window,sink", [(1, 0), (1, 1), (5, 3), (16, 16), (64, 0), (100, 20), (333, 100), (5000, 7), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (3, 3)])
def test_windows(hq, hkv, window, sink):
    c = Case(2, MIXED, hq, hkv, HND if hkv == 2 else NHD, window=window, sink=sink)
    c.check(*c.call())


@pytest.mark.parametrize("n,ctx", [(1, 1), (2, 2), (15, 15), (16, 16), (17, 17), (79, 80), (80, 80), (81, 81), (1, 81), (32, 160), (33, 161), (64, 400), (127, 127),
                                   (129, 129), (255, 300), (257, 257), (640, 641)])
def test_single_sequences(n, ctx):
    c = Case(3, [(n, ctx)], 8, 2, behind=0)
    c.check(*c.call())


def test_a_long_context_is_cut_over_the_device():
    for n in (1, 3, 40, 70):
        c = Case(4, [(n, 40013)], 4, 1)
        c.check(*c.call())


def test_rows_before_the_first_token_see_nothing():
    c = Case(5, [(7, 3), (1, 30), (300, 100), (4, 0)], 8, 2)
    out, lse = c.call()
    c.check(out, lse)
    assert bool((out[:4] == 0).all()) and bool((lse[:4] == -torch.inf).all())


@pytest.mark.parametrize("hq,hkv", [(8, 8), (16, 1)])
def test_more_units_than_one_round_plans(hq, hkv):
    rng = np.random.default_rng(6)
    many = 148 * 80 // hkv + 50 if hkv > 1 else 3000
    c = Case(6, [(int(n), int(n + x)) for n, x in zip(rng.integers(0, 3, many), rng.integers(0, 20, many))], hq, hkv)
    out, lse = c.call()
    c.check(out, lse, only=[0, 1, 2, many // 2, many // 2 + 1, many - 2, many - 1] + list(rng.integers(0, many, 60)))
    assert not bool(out[:int(c.q_indptr[-1])].isnan().any())


def test_scores_that_rise_and_fall():
    # spread over hundreds of units of the exponent: the reference moves in many steps, early weights vanish
    c = Case(7, [(100, 900), (1, 3000), (20, 20)], 8, 2, hot=40.0)
    c.check(*c.call())
    c = Case(8, [(100, 900), (1, 3000), (20, 20)], 8, 2, hot=40.0, window=200, sink=4)
    c.check(*c.call())


def test_scales():
    for scale in (1e-6, 1.0):
        c = Case(9, [(70, 300), (1, 500)], 8, 2, scale=scale)
        c.hot = max(1.0, scale / D ** -0.5)
        c.check(*c.call())


# A sequence alone behind a context whose K and V are too much for the caches is divided differently (all CTAs walk it together): from 48 MiB on, 8 KV
# heads that is 12288 tokens, and with at least eight tokens for each row.
@pytest.mark.parametrize("n,ctx,hq,hkv,window,sink", [
    (70, 12300, 32, 8, 0, 0),          # 2 tiles a head, 16 units: none whole
    (1100, 13001, 32, 8, 0, 0),        # 18 tiles, 144 units
    (1500, 12777, 32, 8, 0, 0),        # 24 tiles, 192 units: one round of whole units, 44 cut
    (300, 20001, 8, 8, 13000, 21),     # through a window of that size
    (513, 13000, 64, 8, 0, 0),         # 17 tiles, 136 units, the last tile one row
    (40, 100003, 16, 1, 0, 0),
])
def test_a_long_context_that_all_walk_together(n, ctx, hq, hkv, window, sink):
    for layout in (HND, NHD):
        c = Case(30, [(0, 100), (n, ctx), (0, 0)], hq, hkv, layout, window=window, sink=sink, before=1)
        out, lse = c.call()
        # in pieces: the whole in 64 bits would not fit
        c.check(out, lse, rows=40 if ctx * hq > 200000 else None)


@pytest.mark.parametrize("layout", [HND, NHD])
@pytest.mark.parametrize("sequences,hq,hkv,window,sink", [
    ([(3600, 3600)], 32, 8, 0, 0), ([(3567, 3600)], 32, 8, 0, 0), ([(2000, 2000), (0, 30), (1801, 1801), (0, 0), (77, 200), (1, 700)], 32, 8, 0, 0),
    ([(1200, 1300), (700, 3000), (2000, 1990), (33, 33)], 32, 8, 200, 10), ([(130 + 97 * i, 130 + 98 * i) for i in range(16)], 16, 4, 0, 0),
    ([(130 + 97 * i, 130 + 98 * i) for i in range(17)], 16, 4, 0, 0), ([(0, 5)] * 360 + [(2500, 2500), (1100, 1100)], 32, 8, 0, 0), ([(4000, 4000), (3900, 3900)], 16, 1, 0, 0),
    ([(4500, 4500), (1000, 1000)], 24, 24, 0, 0),
])
def test_many_whole_units(sequences, hq, hkv, window, sink, layout):
    # prompts whose units are dealt out whole, on both sides of the limits of that
    c = Case(40 + len(sequences), sequences, hq, hkv, layout, window=window, sink=sink)
    out, lse = c.call()
    c.check(out, lse, rows=150)


def test_more_dealt_units_than_one_round_plans():
    # 64 heads of 176 tiles, 76 units a CTA
    c = Case(45, [(45056, 45056)], 64, 64, window=300, sink=3)
    out, lse = c.call()
    c.check(out, lse, rows=64)
    again = c.call()
    assert torch.equal(out.view(torch.int16), again[0].view(torch.int16)) and torch.equal(lse.view(torch.int32), again[1].view(torch.int32))


def test_agrees_with_verify_attn():
    c = Case(10, [(4, 700), (1, 33), (8, 2000)], 8, 2, behind=0)
    out, lse = c.call()
    ws = kap.Workspace(max_rows_per_item=32, max_batch=3)
    ws.schedule((c.ctx + PAGE - 1) // PAGE, c.n_q, 8, 2)
    ref, ref_lse = torch.empty_like(out), torch.empty_like(lse)
    kap.verify_attn(c.q, gu.i32(c.q_indptr), c.pool, gu.i32(c.bt_indptr), gu.i32(c.bt), gu.i32(c.ctx), ref, ws, lse=ref_lse)
    ws.check()
    c.check(out, lse)
    # verify_attn sums the weights after their rounding to bf16, at most 2^-8 of each: its lse is off by up to ln(1 + 2^-8)
    assert float((lse - ref_lse).abs().max()) < 2.0 ** -8 + 2e-5
    # each result is within a rounding of the weights (2^-8 of the weighted mean of |V|; verify_attn's are normalised by the rounded sum: twice that)
    # and of the result
    size = torch.cat([c.expected(b)[2] for b in range(3)])
    assert bool(((out.double() - ref.double()).abs() <= 3 * 2.0 ** -8 * size + 2.0 ** -7 * ref.double().abs() + 4e-4 * size).all())


def test_the_layouts_hold_the_same_values():
    a = Case(11, MIXED, 8, 2, HND, window=90, sink=5)
    b = Case(11, MIXED, 8, 2, NHD, window=90, sink=5)
    b.pool.copy_(a.pool.transpose(2, 3))
    for x, y in zip(a.call(), b.call()):
        assert torch.equal(x.nan_to_num(7.0), y.nan_to_num(7.0))


def test_calls_repeat_and_need_no_lse():
    c = Case(12, MIXED, 8, 2)
    out, lse = c.call()
    again, _ = c.call()
    assert torch.equal(out.nan_to_num(7.0), again.nan_to_num(7.0))
    bare = torch.full_like(c.q, float("nan"))
    kap.chunk_attn(c.q, gu.i32(c.q_indptr), c.pool, gu.i32(c.bt_indptr), gu.i32(c.bt), gu.i32(c.ctx), bare, c.ws)
    assert torch.equal(out.nan_to_num(7.0), bare.nan_to_num(7.0))


def test_captured_calls_follow_the_lengths():
    big = Case(13, [(100, 900), (30, 600), (1, 400)], 8, 2, behind=0)
    steps = [(np.array([100, 30, 1]), big.ctx), (np.array([1, 1, 1]), np.array([500, 16, 400])), (np.array([0, 90, 3]), np.array([800, 599, 17])),
             (np.array([0, 0, 0]), np.array([1, 2, 3]))]
    indptr, ctx = gu.i32(big.q_indptr), gu.i32(big.ctx)
    bt = gu.i32(big.bt_indptr), gu.i32(big.bt)
    out, lse = torch.empty_like(big.q), torch.empty(big.q.shape[:2], device=gu.DEV)
    ws = big.workspace()
    call = lambda o, l, w: kap.chunk_attn(big.q, indptr, big.pool, *bt, ctx, o, w, lse=l)      # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out, lse, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, lse, ws)
    eager_ws = big.workspace()
    for n_q, lengths in steps + steps[::-1]:
        big.n_q, big.ctx, big.q_indptr = n_q, lengths, np.concatenate([[0], np.cumsum(n_q)])
        indptr.copy_(gu.i32(big.q_indptr))
        ctx.copy_(gu.i32(lengths))
        out.fill_(float("nan")), lse.fill_(float("nan"))
        graph.replay()
        ws.check()
        big.check(out, lse)
        o, l = torch.full_like(out, float("nan")), torch.full_like(lse, float("nan"))
        call(o, l, eager_ws)
        eager_ws.check()
        assert torch.equal(out.nan_to_num(7.0), o.nan_to_num(7.0)) and torch.equal(lse.nan_to_num(7.0), l.nan_to_num(7.0))


def test_two_streams_with_a_workspace_each():
    cases = [Case(14 + i, [(200, 3000), (1, 5000), (64, 64)], 8, 2) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    for c in cases:
        c.ws = c.workspace()
    torch.cuda.synchronize()
    results = []
    for _ in range(3):
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                results.append((c, c.call(check=False)))
    torch.cuda.synchronize()
    for c, r in results:
        c.ws.check()
        c.check(*r)


def test_a_schedule_of_the_workspace_stays():
    c = Case(16, [(4, 700), (1, 33)], 8, 2, behind=0)
    ws = c.workspace()
    ws.schedule((c.ctx + PAGE - 1) // PAGE, c.n_q, 8, 2)
    args = c.q, gu.i32(c.q_indptr), c.pool, gu.i32(c.bt_indptr), gu.i32(c.bt), gu.i32(c.ctx)
    first, second = torch.empty_like(c.q), torch.empty_like(c.q)
    kap.verify_attn(*args, first, ws)
    c.check(*c.call(ws))
    kap.verify_attn(*args, second, ws)
    ws.check()
    assert torch.equal(first, second)


def test_pages_past_32_bit_offsets():
    c = Case(17, [(40, 500), (1, 200)], 16, 8, pages=70000)          # 4.6 GB; the used pages are the last ones
    assert int(c.bt.max()) * 2 * 8 * PAGE * D > 2 ** 31
    c.check(*c.call())
    c = Case(18, [(40, 500), (1, 200)], 16, 8, NHD, pages=70000)
    c.check(*c.call())


def _reported(c, **change):
    for name, value in change.items():
        setattr(c, name, value)
    out, lse = c.call(check=False)
    with pytest.raises(kap.KapError) as e:
        c.ws.check()
    assert e.value.code == kap.ERR_DEVICE_INDEX
    return out, lse


def test_bad_pages_and_lengths_are_reported():
    sequences = [(20, 300), (40, 200), (1, 90)]
    for bad in (-1, 10 ** 6):
        c = Case(19, sequences, 8, 2)
        bt = c.bt.copy()
        bt[c.bt_indptr[1] + 3] = bad
        good, c.bt = c.bt, bt
        heads = c.heads_first()
        heads[0] = 0.25                                               # page 0 is read in its place
        out, lse = _reported(c)
        c.bt = good
        c.check(out, lse, only=[0, 2])
    # a context beyond its block table, a negative one
    for length in (10 ** 6, -5):
        c = Case(20, sequences, 8, 2)
        good, ctx = c.ctx, c.ctx.copy()
        ctx[0] = length
        out, lse = _reported(c, ctx=ctx)
        c.ctx = good
        c.check(out, lse, only=[1, 2])
    # rows that q does not have, offsets that fall
    for indptr in ([0, 20, 60, 1000], [0, 20, 10, 61], [-4, 20, 60, 61]):
        c = Case(21, sequences, 8, 2, behind=0)
        _reported(c, q_indptr=np.array(indptr, dtype=np.int32))
        torch.cuda.synchronize()


@pytest.mark.parametrize("sequences,hq,hkv", [([(300, 700), (1, 5000), (40, 40)], 8, 2), ([(50, 4000)], 8, 2), ([(150, 150)], 2, 2), ([(1, 20000)], 16, 1)])
def test_a_query_with_nan_gets_nan_alone(sequences, hq, hkv):
    # in units of one CTA and in cut ones, of a pair, of one tile and of 64 rows
    c = Case(33, sequences, hq, hkv)
    good, good_lse = c.call()
    rows = torch.tensor([int(c.q_indptr[b]) + int(n) - 1 for b, (n, _) in enumerate(sequences)] + [int(c.q_indptr[0])], device=gu.DEV)
    c.q[rows, 1, 5] = float("nan")
    out, lse = c.call()
    hit = torch.zeros(c.rows, hq, dtype=torch.bool, device=gu.DEV)
    hit[rows, 1] = True
    assert bool(out[hit].isnan().all()) and bool(lse[hit].isnan().all())
    used = slice(int(c.q_indptr[0]), int(c.q_indptr[-1]))
    keep = ~hit[used]
    assert torch.equal(out[used][keep], good[used][keep]) and torch.equal(lse[used][keep], good_lse[used][keep])


def _repeated(tokens, listed=None, hq=1, list0=0):
    """one token after `tokens` - 1 others in a cache whose block table names one page again and again; keys 0, values 1, 2, 4, ..."""
    pool = torch.zeros((2, 2, 1, PAGE, D), dtype=torch.bfloat16, device=gu.DEV)
    value = 2.0 ** (torch.arange(D, device=gu.DEV) % 8)
    pool[1, 1] = value.to(torch.bfloat16)
    table = torch.ones((listed or tokens + PAGE - 1) // PAGE, dtype=torch.int32, device=gu.DEV)
    q = torch.ones((1, hq, D), dtype=torch.bfloat16, device=gu.DEV)
    out, lse = torch.full_like(q, float("nan")), torch.full((1, hq), float("nan"), device=gu.DEV)
    ws = kap.Workspace(max_items=kap.chunk_attn_items(), max_rows_per_item=64, max_batch=1)
    kap.chunk_attn(q, gu.i32([0, 1]), pool, gu.i32([list0, list0 + len(table)]), table, gu.i32([tokens]), out, ws, lse=lse)
    return ws, out, lse, value


def test_the_longest_context():
    # weights of 1, whose partial sums are whole numbers below 2^24: only lse is rounded (a logarithm of 2^26, 18.02: three roundings of 2^-24 of it)
    ws, out, lse, value = _repeated(2 ** 26)
    ws.check()
    assert torch.equal(out[0, 0].float(), value)
    assert abs(float(lse[0, 0]) - 26 * np.log(2.0)) <= 4e-6


@pytest.mark.parametrize("tokens,list0", [(2 ** 26 + 1, 0), (100, -1), (100, -2 ** 31)])
def test_lengths_and_lists_that_are_not_followed(tokens, list0):
    ws, *_ = _repeated(tokens, list0=list0)
    with pytest.raises(kap.KapError) as e:
        ws.check()
    assert e.value.code == kap.ERR_DEVICE_INDEX
    ws.check()


def test_refusals():
    c = Case(22, [(4, 40)], 8, 2)
    small = kap.Workspace(max_items=10, max_rows_per_item=64, max_batch=4)
    with pytest.raises(kap.KapError) as e:
        c.call(small)
    assert e.value.code == kap.ERR_CAPACITY
    few = kap.Workspace(max_items=kap.chunk_attn_items(), max_rows_per_item=64, max_batch=1)
    with pytest.raises(kap.KapError) as e:
        Case(22, [(4, 40), (1, 2)], 8, 2).call(few)
    assert e.value.code == kap.ERR_CAPACITY
    ws = c.workspace()
    args = [c.q, gu.i32(c.q_indptr), c.pool, gu.i32(c.bt_indptr), gu.i32(c.bt), gu.i32(c.ctx), torch.empty_like(c.q), ws]
    for kw, code in ((dict(window=-1), kap.ERR_INVALID_ARG), (dict(n_sink=-1), kap.ERR_INVALID_ARG), (dict(sm_scale=0.0), kap.ERR_INVALID_ARG),
                     (dict(sm_scale=float("nan")), kap.ERR_INVALID_ARG), (dict(lse=torch.empty(3, 8, device=gu.DEV)), kap.ERR_INVALID_ARG)):
        with pytest.raises(kap.KapError) as e:
            kap.chunk_attn(*args, **kw)
        assert e.value.code == code
    for i, bad in ((0, c.q.float()), (0, c.q[:, ::2]), (0, c.q.cpu()), (1, gu.i32(c.q_indptr).long()), (1, gu.i32(c.q_indptr)[:1]), (2, c.pool[:, :, :, :, ::2]),
                   (6, torch.empty_like(c.q[1:])), (0, torch.empty((7, 6, D), dtype=torch.bfloat16, device=gu.DEV))):
        changed = list(args)
        changed[i] = bad
        if i == 0 and bad.shape[1] == 6:
            changed[6] = torch.empty_like(bad)
        with pytest.raises(kap.KapError):
            kap.chunk_attn(*changed)
