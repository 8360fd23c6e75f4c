"""kap_shared_prefix_attn on the GPU against plain attention in 64 bits, and against kap_verify_attn on the same arrays.

Tolerance of a result: each weight is rounded to bf16 for the product with V (at most 2^-8 of it), so the weighted mean moves by at
most 2^-8 of the weighted mean of |V|; a score is a fp32 sum of 128 products, off by less than 128 2^-24 sum |q k| scale (below 1e-4 for
these inputs), which moves a weight by as much of itself; the result is rounded to bf16 once (2^-8 of it).
lse: the same 1e-4 bounds its absolute error; the typical one is 1e-6, and 2e-5 absolute is asked for (an average over the row's scores)."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap

pytestmark = pytest.mark.gpu
D, PAGE = 128, 16


class Case:
    """groups: a list of (prefix pages, [(n_q, own tokens), ...])"""

    def __init__(self, seed, groups, hq=8, hkv=2, layout=kap.KV_HND, spare=0, scale=None, poison=float("nan")):
        g = torch.Generator(device=gu.DEV).manual_seed(seed)
        self.hq, self.hkv, self.layout, self.scale = hq, hkv, layout, D ** -0.5 if scale is None else scale
        self.prefix = np.array([p for p, _ in groups], dtype=np.int32)
        members = [len(m) for _, m in groups]
        self.cuts = np.concatenate([[0], np.cumsum(members)]).astype(np.int32)
        self.group = np.repeat(np.arange(len(groups)), members)
        self.n_q = np.array([q for _, m in groups for q, _ in m], dtype=np.int32)
        self.tail = np.array([t for _, m in groups for _, t in m], dtype=np.int64)
        self.ctx = (self.prefix[self.group] * PAGE + self.tail).astype(np.int32)
        own = (self.tail + PAGE - 1) // PAGE + spare
        self.lists = (self.prefix[self.group] + own).astype(np.int32)
        self.lists[self.lists == 0] = 1
        own = self.lists - self.prefix[self.group]
        n_pages = int(self.prefix.sum() + own.sum()) + 2
        perm = np.random.default_rng(seed).permutation(n_pages)
        shared, at = [], 0
        for p in self.prefix:
            shared.append(perm[at:at + p])
            at += p
        table = []
        for b in range(len(self.n_q)):
            table += [shared[self.group[b]], perm[at:at + own[b]]]
            at += own[b]
        self.bt = np.concatenate(table).astype(np.int32)
        self.bt_indptr = np.concatenate([[0], np.cumsum(self.lists)]).astype(np.int32)
        self.q_indptr = np.concatenate([[0], np.cumsum(self.n_q)]).astype(np.int32)
        shape = (n_pages, 2, hkv, PAGE, D) if layout == kap.KV_HND else (n_pages, 2, PAGE, hkv, D)
        self.pool = (torch.randn(shape, device=gu.DEV, generator=g) * 0.5).to(torch.bfloat16)
        self.q = torch.randn((int(self.n_q.sum()), hq, D), device=gu.DEV, generator=g).to(torch.bfloat16)
        # everything behind the contexts holds `poison`
        heads = self.heads_first()
        used = torch.zeros(n_pages, PAGE, dtype=torch.bool, device=gu.DEV)
        for b in range(len(self.n_q)):
            t = np.arange(self.ctx[b])
            used[torch.from_numpy(self.bt[self.bt_indptr[b] + t // PAGE].astype(np.int64)).to(gu.DEV), torch.from_numpy(t % PAGE).to(gu.DEV)] = True
        heads[(~used)[:, None, None, :].expand(-1, 2, hkv, -1)] = poison
        self.ws = None

    def heads_first(self):
        return self.pool if self.layout == kap.KV_HND else self.pool.transpose(2, 3)

    def workspace(self):
        args = self.lists, self.n_q, self.cuts, self.prefix, self.hq, self.hkv
        ws = kap.Workspace(max_items=kap.shared_prefix_items(*args), max_rows_per_item=64, max_batch=len(self.n_q))
        ws.set_kv_layout(self.layout)
        ws.schedule_shared_prefix(*args)
        return ws

    def arrays(self, ctx=None):
        return self.q, gu.i32(self.q_indptr), self.pool, gu.i32(self.bt_indptr), gu.i32(self.bt), gu.i32(self.ctx if ctx is None else ctx)

    def call(self, ctx=None, ws=None):
        self.ws = ws or self.ws or self.workspace()
        out = torch.full_like(self.q, float("nan"))
        lse = torch.full(self.q.shape[:2], float("nan"), device=gu.DEV)
        kap.shared_prefix_attn(*self.arrays(ctx), out, self.ws, lse=lse, sm_scale=self.scale)
        self.ws.check()
        return out, lse

    def reference(self, ctx=None):
        """out, lse and the weighted mean of |V|, in 64 bits"""
        ctx = self.ctx if ctx is None else np.asarray(ctx)
        share, heads = self.hq // self.hkv, self.heads_first()
        out = torch.zeros(self.q.shape, dtype=torch.float64, device=gu.DEV)
        size, lse = torch.zeros_like(out), torch.full(self.q.shape[:2], -np.inf, dtype=torch.float64, device=gu.DEV)
        for b in range(len(self.n_q)):
            L, r0, r1 = int(ctx[b]), int(self.q_indptr[b]), int(self.q_indptr[b + 1])
            pages = torch.from_numpy(self.bt[self.bt_indptr[b]:self.bt_indptr[b + 1]].astype(np.int64)).to(gu.DEV)
            kv = heads[pages].double()                                        # [pages, 2, Hkv, 16, D]
            k, v = (kv[:, i].transpose(0, 1).flatten(1, 2)[:, :max(L, 0)] for i in (0, 1))
            q = self.q[r0:r1].double().view(r1 - r0, self.hkv, share, D) * self.scale
            z = torch.einsum("rhgd,htd->rhgt", q, k)
            for j in range(r1 - r0):
                n = L - (r1 - r0) + j + 1
                if n <= 0:
                    continue
                row = z[j, :, :, :n]
                lse[r0 + j] = row.logsumexp(-1).flatten()
                w = row.softmax(-1)
                out[r0 + j] = torch.einsum("hgt,htd->hgd", w, v[:, :n]).flatten(0, 1)
                size[r0 + j] = torch.einsum("hgt,htd->hgd", w, v[:, :n].abs()).flatten(0, 1)
        return out, lse, size

    def check(self, ctx=None, ws=None):
        got, lse = self.call(ctx, ws)
        out, ref, size = self.reference(ctx)
        over = ((got.double() - out).abs() - (2.0 ** -8 + 1e-4) * size - 2.0 ** -8 * out.abs()).max().item()
        assert over <= 1e-30, f"off by {over} more than allowed"
        empty = ref == -np.inf
        assert torch.equal(lse == -np.inf, empty) and (got[empty] == 0).all()
        err = (lse.double() - ref)[~empty].abs()
        assert err.numel() == 0 or err.max().item() <= 2e-5, f"lse off by {err.max().item()}"
        return got, lse


@pytest.mark.parametrize("layout", [kap.KV_HND, kap.KV_NHD])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (4, 2), (8, 2), (16, 2), (16, 1), (32, 8)])
def test_head_groups_and_layouts(hq, hkv, layout):
    Case(1, [(9, [(1, 5), (3, 40), (1, 1), (2, 130)]), (0, [(1, 77)])], hq, hkv, layout).check()


@pytest.mark.parametrize("prefix", [0, 1, 3, 4, 5, 7, 8, 9, 31, 64, 65])
def test_prefix_lengths(prefix):
    Case(2, [(prefix, [(1, 3), (1, 64), (4, 65), (1, 16)])]).check()


@pytest.mark.parametrize("tail", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 1000])
def test_own_lengths(tail):
    Case(3, [(6, [(1, tail), (1, 1)]), (2, [(min(tail, 8), tail)])]).check()


@pytest.mark.parametrize("members,n_q", [(2, 1), (31, 1), (32, 1), (33, 1), (64, 1), (65, 1), (130, 1), (40, 8), (5, 16), (17, 3)])
def test_rows_of_a_group(members, n_q):
    rng = np.random.default_rng(members)
    Case(4, [(21, [(n_q, int(t)) for t in rng.integers(n_q, 90, members)])], hq=8, hkv=2).check()


def test_many_groups_of_many_shapes():
    rng = np.random.default_rng(5)
    groups = [(int(rng.integers(0, 60)), [(int(rng.integers(1, 9)), int(rng.integers(9, 300))) for _ in range(int(rng.integers(1, 9)))])
              for _ in range(11)]
    for layout in (kap.KV_HND, kap.KV_NHD):
        Case(5, groups, 16, 4, layout).check()


def test_long_prefix():
    Case(6, [(2050, [(1, 30), (2, 700), (1, 16), (5, 5)])], 32, 8).check()
    Case(7, [(700, [(4, 40 + 3 * i) for i in range(48)])], 32, 8).check()


@pytest.mark.parametrize("layout", [kap.KV_HND, kap.KV_NHD])
@pytest.mark.parametrize("members", [17, 18, 24, 33, 39, 45, 70, 72, 97])
def test_partly_filled_tiles_over_many_steps(members, layout):
    # 68 rows (one tile) to 388 (a pair and a single tile): softmax warps with all, some and none of their rows
    rng = np.random.default_rng(members)
    Case(30, [(403, [(1, int(t)) for t in rng.integers(1, 60, members)]), (130, [(1, int(t)) for t in rng.integers(1, 60, 20)])], 8, 2, layout).check()


@pytest.mark.parametrize("layout", [kap.KV_HND, kap.KV_NHD])
@pytest.mark.parametrize("prefix", [0, 33])
def test_crowded_batches(prefix, layout):
    # more short own parts than CTAs fit the device at once, with some long ones and some windows of many rows among them
    rng = np.random.default_rng(prefix)
    members = [(int(rng.integers(1, 5)), int(t)) for t in rng.integers(4, 300, 62)] + [(1, 1), (1, 2000), (16, 40), (9, 790), (4, 768), (1, 769)]
    Case(31, [(prefix, members)], 32, 8, layout).check()


def test_windows_longer_than_the_own_part():
    # a sequence whose rows reach back into the shared pages, and one with nothing of its own
    Case(8, [(4, [(3, 1), (1, 0), (6, 2), (1, 9)])]).check()


def test_contexts_shorter_and_longer_than_scheduled():
    c = Case(9, [(5, [(1, 40), (2, 90), (3, 17)]), (0, [(2, 50)])], spare=4, poison=0.25)
    for ctx in (c.ctx, c.ctx + 30, c.ctx - 16, [80, 81, 82, 2], [64, 3, 1, 1], [1, 1, 1, 1], [0, 2, 0, 0], c.lists * PAGE):
        c.check(ctx)


def test_rows_that_see_nothing():
    c = Case(10, [(0, [(3, 2), (1, 1)]), (0, [(8, 3), (1, 0)])], poison=0.0)
    got, lse = c.check()
    assert (lse[0] == -np.inf).all() and (got[0] == 0).all() and (lse[-1] == -np.inf).all()


def test_scores_of_every_size():
    for scale in (1e-6, 0.7, 30.0):
        c = Case(11, [(40, [(1, 200), (2, 3)])], scale=scale)
        got, lse = c.call()
        out, ref, size = c.reference()
        # a score of magnitude z carries a fp32 error of about 2^-21 z, which moves its weight by as much of itself
        z = 128 * 1.2 * scale
        assert ((got.double() - out).abs() <= (2.0 ** -8 + 1e-4 + 2.0 ** -17 * z) * size * 2 + 2.0 ** -8 * out.abs() + 1e-30).all()
        assert ((lse.double() - ref).abs() <= 2e-5 + 2.0 ** -20 * z).all()


def test_running_maximum_that_keeps_rising():
    # keys that grow along the context: every tile lifts the reference of the exponentials
    c = Case(12, [(64, [(1, 300), (4, 90)])])
    heads = c.heads_first()
    for b in range(2):
        pages = c.bt[c.bt_indptr[b]:c.bt_indptr[b + 1]]
        for i, page in enumerate(pages):
            heads[int(page), 0] = (c.q[0, 0].float() * 0.02 * (i + 1)).to(torch.bfloat16)
    got, lse = c.call()
    out, ref, size = c.reference()
    assert ((got.double() - out).abs() <= (2.0 ** -8 + 2e-3) * size + 2.0 ** -8 * out.abs() + 1e-30).all()
    assert ((lse.double() - ref).abs() <= 2.0 ** -20 * ref.abs() + 2e-5).all()


def test_equal_to_verify_attn_on_the_same_arrays():
    c = Case(13, [(30, [(4, 40), (5, 100), (4, 33)]), (12, [(1, 5), (8, 8)])], 32, 8, poison=0.0)
    out, lse = c.call()
    ws = kap.Workspace(max_rows_per_item=64, max_batch=5)
    ws.schedule((c.ctx + PAGE - 1) // PAGE, c.n_q, c.hq, c.hkv)
    want, want_lse = torch.empty_like(out), torch.empty_like(lse)
    kap.verify_attn(*c.arrays(), want, ws, lse=want_lse, sm_scale=c.scale)
    ws.check()
    # verify_attn's own error is as large, and its lse sums rounded weights (2^-8 of each)
    _, _, size = c.reference()
    assert ((out.double() - want.double()).abs() <= 2 * (2.0 ** -8 + 1e-4) * size + 2 * 2.0 ** -8 * want.double().abs()).all()
    assert (lse - want_lse).abs().max().item() <= 2.0 ** -8


def test_one_workspace_for_both_schedules_in_turn():
    c = Case(14, [(20, [(4, 40), (4, 50)])], poison=0.0)
    ws = kap.Workspace(max_items=2048, max_rows_per_item=64, max_batch=2)
    ws.schedule_shared_prefix(c.lists, c.n_q, c.cuts, c.prefix, c.hq, c.hkv)
    args = (c.ctx + PAGE - 1) // PAGE, c.n_q, c.hq, c.hkv
    out = torch.empty_like(c.q)
    with pytest.raises(kap.KapError) as e:
        kap.verify_attn(*c.arrays(), out, ws)
    assert e.value.code == kap.ERR_INVALID_ARG
    first = c.check(ws=ws)
    ws.schedule(*args)
    with pytest.raises(kap.KapError) as e:
        kap.shared_prefix_attn(*c.arrays(), out, ws)
    assert e.value.code == kap.ERR_INVALID_ARG
    kap.verify_attn(*c.arrays(), out, ws)
    ws.check()
    ws.schedule_shared_prefix(c.lists, c.n_q, c.cuts, c.prefix, c.hq, c.hkv)
    again = c.check(ws=ws)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_refusals():
    c = Case(15, [(3, [(1, 4), (1, 9)])])
    ws = c.workspace()
    out = torch.empty_like(c.q)
    q, qi, pool, bti, btp, ctx = c.arrays()
    for args, kw in (((q[:, :4].contiguous(), qi, pool, bti, btp, ctx), {}), ((q, qi, pool, bti, btp, ctx[:1]), {}),
                     ((q, qi, pool, bti, btp, ctx), dict(sm_scale=0.0)), ((q, qi, pool, bti, btp, ctx), dict(sm_scale=float("nan"))),
                     ((q, qi, pool, bti, btp, ctx), dict(sm_scale=-1.0))):
        with pytest.raises(kap.KapError):
            kap.shared_prefix_attn(*args, out, ws, **kw)
    small = kap.Workspace(max_items=1, max_rows_per_item=1, max_batch=2)
    big = Case(16, [(300, [(4, 400)] * 2)])
    with pytest.raises(kap.KapError) as e:
        small.schedule_shared_prefix(big.lists, big.n_q, big.cuts, big.prefix, big.hq, big.hkv)
    assert e.value.code == kap.ERR_CAPACITY
    with pytest.raises(kap.KapError) as e:
        small.schedule_shared_prefix([4] * 3, [1] * 3, [0, 3], [2], 8, 2)
    assert e.value.code == kap.ERR_CAPACITY
    c.check(ws=ws)


def test_bad_pages_are_reported():
    for bad in (-1, 10 ** 6):
        for at in (1, -1):
            c = Case(17, [(3, [(1, 40), (1, 9)])], poison=0.0)
            table = c.bt.copy()
            table[at] = bad
            q, qi, pool, bti, _, ctx = c.arrays()
            ws = c.workspace()
            kap.shared_prefix_attn(q, qi, pool, bti, gu.i32(table), ctx, torch.empty_like(c.q), ws)
            with pytest.raises(kap.KapError) as e:
                ws.check()
            assert e.value.code == kap.ERR_DEVICE_INDEX
            ws.check()                                                           # reading the status clears it


def test_runs_repeat_bit_for_bit():
    c = Case(18, [(90, [(2, 40 + i) for i in range(20)])], 32, 8)
    first = c.call()
    for _ in range(4):
        again = c.call()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_graph_capture_and_two_workspaces_on_two_streams():
    cases = [Case(20 + i, [(50, [(1, 60), (3, 33)]), (7, [(2, 20)])]) for i in range(2)]
    want = [c.call() for c in cases]
    c = cases[0]
    arrays, out = c.arrays(), torch.zeros_like(c.q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kap.shared_prefix_attn(*arrays, out, c.ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0][0])
    streams, outs, args = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(x.q) for x in cases], [x.arrays() for x in cases]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                kap.shared_prefix_attn(*args[i], outs[i], cases[i].ws)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], want[i][0])


def test_rows_behind_the_last_sequence_are_left_alone():
    c = Case(22, [(6, [(1, 20), (2, 9)])])
    want, _ = c.call()
    q = torch.cat([c.q, c.q[:2]])
    out = torch.full_like(q, 3.0)
    _, qi, pool, bti, btp, ctx = c.arrays()
    kap.shared_prefix_attn(q, qi, pool, bti, btp, ctx, out, c.ws)
    c.ws.check()
    assert torch.equal(out[:3], want) and (out[3:] == 3.0).all()
