"""kap_build_block_tables and kap_release_pages on the GPU against a plain program on the host; everything is a whole number and has to be equal."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap

pytestmark = pytest.mark.gpu


class Server:
    """requests with their pages, kept twice: on the device by the calls, on the host by the rules"""

    def __init__(self, requests, wide, pages, seed=0, page=16, spare=0):
        rng = np.random.default_rng(seed)
        self.page, self.wide = page, wide
        self.table = np.full((requests, wide), -1, dtype=np.int32)
        self.held = np.zeros(requests, dtype=np.int32)
        self.free = np.concatenate([rng.permutation(pages), np.full(spare, -1)]).astype(np.int32)
        self.count = pages
        self.dev = dict(page_table=gu.i32(self.table), pages_held=gu.i32(self.held), free_pages=gu.i32(self.free), free_count=gu.i32([self.count]))
        self.status = torch.zeros(1, dtype=torch.int32, device=gu.DEV)

    def build(self, ctx, n_new=None, request=None, capacity=None, rows=None, lists=True):
        batch = len(ctx)
        req = np.arange(batch) if request is None else np.asarray(request)
        new = np.ones(batch, dtype=np.int64) if n_new is None else np.asarray(n_new, dtype=np.int64)
        pages = (np.asarray(ctx, dtype=np.int64) + new + self.page - 1) // self.page
        capacity = int(pages.sum()) + 5 if capacity is None else capacity
        rows = int(new.sum()) + 3 if rows is None else rows
        out = dict(bt_indptr=torch.full((batch + 1,), -9, dtype=torch.int32, device=gu.DEV), bt_pages=torch.full((capacity,), -9, dtype=torch.int32, device=gu.DEV),
                   new_indptr=torch.full((batch + 1,), -9, dtype=torch.int32, device=gu.DEV), slot=torch.full((rows,), -9, dtype=torch.int64, device=gu.DEV),
                   position=torch.full((rows,), -9, dtype=torch.int32, device=gu.DEV))
        kap.build_block_tables(gu.i32(ctx), **self.dev, n_new=None if n_new is None else gu.i32(n_new), request=None if request is None else gu.i32(request),
                               page_size=self.page, device_status=self.status, **out)
        return {k: v.cpu().numpy() for k, v in out.items()}, pages, new, req

    def expect_build(self, got, ctx, pages, new, req):
        for b, r in enumerate(req):
            for i in range(self.held[r], pages[b]):
                self.count -= 1
                self.table[r, i] = self.free[self.count]
            self.held[r] = max(self.held[r], pages[b])
        assert np.array_equal(got["bt_indptr"], np.concatenate([[0], np.cumsum(pages)]))
        assert np.array_equal(got["new_indptr"], np.concatenate([[0], np.cumsum(new)]))
        lists = np.concatenate([self.table[r, :n] for r, n in zip(req, pages)] + [np.full(len(got["bt_pages"]) - pages.sum(), -9)])
        assert np.array_equal(got["bt_pages"], lists)
        pos = [np.arange(c, c + n) for c, n in zip(ctx, new)]
        slot = [self.table[r, p // self.page].astype(np.int64) * self.page + p % self.page for r, p in zip(req, pos)]
        rest = np.full(len(got["slot"]) - new.sum(), -9)
        assert np.array_equal(got["position"], np.concatenate(pos + [rest]))
        assert np.array_equal(got["slot"], np.concatenate(slot + [rest]))
        self.expect_state()

    def step(self, ctx, n_new=None, request=None):
        got, *rest = self.build(ctx, n_new, request)
        assert int(self.status[0]) == 0
        self.expect_build(got, ctx, *rest)

    def expect_state(self):
        assert np.array_equal(self.dev["page_table"].cpu().numpy(), self.table)
        assert np.array_equal(self.dev["pages_held"].cpu().numpy(), self.held)
        assert np.array_equal(self.dev["free_pages"].cpu().numpy()[:self.count], self.free[:self.count])
        assert int(self.dev["free_count"][0]) == self.count

    def release(self, request=None, keep=None):
        kap.release_pages(None if request is None else gu.i32(request), **self.dev, keep_tokens=None if keep is None else gu.i32(keep), page_size=self.page,
                          device_status=self.status)

    def expect_release(self, request=None, keep=None):
        req = np.arange(len(self.held)) if request is None else np.asarray(request)
        moved = []
        for i, r in enumerate(req):
            left = min(self.held[r], 0 if keep is None else (keep[i] + self.page - 1) // self.page)
            moved += list(self.table[r, left:self.held[r]])
            self.held[r] = left
        self.free[self.count:self.count + len(moved)] = moved[::-1]
        self.count += len(moved)
        self.expect_state()


@pytest.mark.parametrize("page", [16, 1, 7, 256])
@pytest.mark.parametrize("batch", [1, 5, 33, 300, 1023, 1025, 2500])
def test_steps_of_a_server(batch, page):
    rng = np.random.default_rng(batch)
    requests = batch + 7
    s = Server(requests, 40 if page > 1 else 220, 300000 if page == 1 else 90000, page=page)
    ctx = np.zeros(batch, dtype=np.int64)
    request = rng.permutation(requests)[:batch]
    for n_new in (rng.integers(0, 120 if page == 1 else 4 * page, batch), None, rng.integers(0, 3, batch), None):
        s.step(ctx, n_new, request)
        ctx += 1 if n_new is None else n_new
    # rejected tokens: the pages stay, and are used again
    ctx = np.maximum(ctx - 2 * page, 0)
    s.step(ctx, None, request)
    # some requests end, others lose their tail; then all goes back
    ended = rng.permutation(request)[:batch // 2 + 1]
    s.release(ended)
    s.expect_release(ended)
    rest = np.setdiff1d(request, ended)
    keep = rng.integers(0, 5 * page, len(rest))
    if len(rest):
        s.release(rest, keep)
        s.expect_release(rest, keep)
    s.release()
    s.expect_release()
    assert s.count == len(s.free) and sorted(s.free) == list(range(len(s.free)))


def test_a_release_undoes_a_step():
    s = Server(20, 100, 2000, seed=3)
    ctx = np.arange(20) * 37
    s.step(ctx)
    state = {k: v.clone() for k, v in s.dev.items()}
    kept = s.free.copy(), s.count, s.held.copy()
    ctx = ctx + 1
    got, *rest = s.build(ctx, np.arange(20) * 11)
    s.expect_build(got, ctx, *rest)
    s.release(None, ctx)
    torch.cuda.synchronize()
    assert all(torch.equal(state[k], s.dev[k]) for k in ("pages_held", "free_count"))
    assert np.array_equal(s.dev["free_pages"].cpu().numpy()[:kept[1]], kept[0][:kept[1]])


def test_long_lists_and_a_long_chunk():
    s = Server(3, 9000, 30000, seed=4)
    s.step([0, 0, 0], [131072, 0, 5])
    s.step([131072, 0, 5], [8000, 100000, 1])


def test_identity_requests_and_no_rows():
    s = Server(6, 10, 50)
    s.step([0, 16, 31, 5, 0, 0], [0, 0, 0, 0, 0, 0])
    assert s.count == 50 - 1 - 2 - 1
    kap.build_block_tables(gu.i32([1, 2]), **s.dev, bt_indptr=(ip := gu.i32([7, 7, 7])), bt_pages=(pg := gu.i32([0] * 4)))      # without the optional arrays
    assert ip.tolist() == [0, 1, 2] and pg.tolist()[:2] == [s.table[0, 0] if s.held[0] else pg.tolist()[0], s.table[1, 0]]


def test_an_empty_step():
    s = Server(6, 10, 50)
    ip, pg, ni = gu.i32([7]), gu.i32([5]), gu.i32([7])
    kap.build_block_tables(gu.i32([]), **s.dev, bt_indptr=ip, bt_pages=pg, new_indptr=ni)
    kap.release_pages(gu.i32([]), **s.dev)
    assert ip.tolist() == [0] and pg.tolist() == [5] and ni.tolist() == [0]
    s.expect_state()


def _refused(s, code, ctx, n_new=None, request=None, **kw):
    s.status.zero_()
    got, *_ = s.build(ctx, n_new, request, **kw)
    assert int(s.status[0]) == code, bin(int(s.status[0]))
    assert not got["bt_indptr"].any() and not got["new_indptr"].any()
    assert (got["bt_pages"] == -9).all() and (got["slot"] == -9).all() and (got["position"] == -9).all()
    s.expect_state()


def test_all_or_nothing():
    full, index = 1 << kap.ERR_CAPACITY, 1 << kap.ERR_DEVICE_INDEX
    for batch in (4, 1500):
        more = batch - 4
        s = Server(batch, 12, 20 + 2 * more)
        tail = [16] * more
        s.step([16, 0, 40, 3] + tail)
        _refused(s, full, [16, 0, 40, 100] + tail, [1, 1, 1, 93] + [1] * more)      # a row of the table: 12 pages, 192 tokens
        _refused(s, full, [16, 0, 40, 100] + tail, [100, 100, 60, 60] + [1] * more)  # the stack
        _refused(s, full, [16, 0, 40, 3] + tail, capacity=6 + 2 * more)              # 2 + 1 + 3 + 1 pages
        _refused(s, full, [16, 0, 40, 3] + tail, [1, 1, 2, 1] + [1] * more, rows=4 + more)
        _refused(s, index, [16, 0, -1, 3] + tail)
        _refused(s, index, [16, 0, 40, 3] + tail, [1, -1, 1, 1] + [1] * more)
        order = np.arange(batch)
        for bad in (-1, batch, 2 ** 31 - 1, 1):                                      # 1: named twice
            request = order.copy()
            request[-1 if bad != 1 else 0] = bad
            _refused(s, index, [16, 0, 40, 3] + tail, None, request)
        _refused(s, full, [2 ** 31 - 1, 0, 40, 3] + tail, [2 ** 31 - 1, 1, 1, 1] + [1] * more, rows=8 + more, capacity=100)
        s.status.zero_()
        s.step([16, 0, 40, 3] + tail)                                                # nothing was lost by any of it
        for name, value in (("free_count", -1), ("free_count", 10 ** 6), ("pages_held", -2), ("pages_held", 13)):
            was = s.dev[name].clone()
            s.dev[name][0] = value
            s.status.zero_()
            got, *_ = s.build([16, 0, 40, 3] + tail)
            assert int(s.status[0]) == index and not got["bt_indptr"].any()
            s.status.zero_()
            s.release()
            assert int(s.status[0]) & index
            s.dev[name].copy_(was)
            s.status.zero_()
        s.expect_state()


def test_a_row_of_the_table_may_be_full():
    s = Server(4, 12, 20)
    s.step([16, 0, 40, 100], [1, 1, 1, 92])                                          # 192 tokens: all 12 pages
    _refused(s, 1 << kap.ERR_CAPACITY, [17, 1, 41, 192])


def test_release_refuses_as_a_whole():
    s = Server(4, 12, 20)
    s.step([16, 0, 40, 3])
    for request in ([0, 1, 0], [0, 4], [-1]):
        s.status.zero_()
        s.release(request)
        assert int(s.status[0]) == 1 << kap.ERR_DEVICE_INDEX
        s.expect_state()
    s.status.zero_()
    s.release([0, 1], [5, -1])
    assert int(s.status[0]) == 1 << kap.ERR_DEVICE_INDEX
    # a stack that cannot take them back
    small = dict(s.dev, free_pages=s.dev["free_pages"][:s.count + 1].clone())
    s.status.zero_()
    kap.release_pages(None, **small, device_status=s.status)
    assert int(s.status[0]) == 1 << kap.ERR_CAPACITY
    s.expect_state()


def test_captured_steps():
    s = Server(8, 64, 600, seed=5)
    ctx, new = gu.i32([0] * 8), gu.i32([1] * 8)
    out = dict(bt_indptr=gu.i32([0] * 9), bt_pages=gu.i32([0] * 600), new_indptr=gu.i32([0] * 9), slot=torch.zeros(400, dtype=torch.int64, device=gu.DEV),
               position=gu.i32([0] * 400))
    start = {k: v.clone() for k, v in s.dev.items()}
    kap.build_block_tables(ctx, **s.dev, n_new=new, **out)
    for k, v in start.items():
        s.dev[k].copy_(v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kap.build_block_tables(ctx, **s.dev, n_new=new, device_status=s.status, **out)
        ctx.add_(new)
    host = np.zeros(8, dtype=np.int64)
    rng = np.random.default_rng(6)
    for k, v in start.items():
        s.dev[k].copy_(v)
    for _ in range(12):
        n = rng.integers(0, 40, 8)
        new.copy_(gu.i32(n))
        for k in ("bt_pages", "slot", "position"):
            out[k].fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.cpu().numpy() for k, v in out.items()}
        s.expect_build(got, host, (host + n + 15) // 16, n, np.arange(8))
        host += n


def test_many_requests():
    s = Server(300000, 2, 5000, seed=7)
    request = np.random.default_rng(8).permutation(300000)[:2000]
    s.step(np.zeros(2000, dtype=np.int64), None, request)
    with pytest.raises(kap.KapError) as e:
        Server(2 ** 20 + 1, 1, 10).step([0])
    assert e.value.code == kap.ERR_UNSUPPORTED


@pytest.mark.parametrize("ctx,new", [(2 ** 31 - 1, 5), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 4, 4)])
def test_a_sequence_of_2_to_the_31_tokens_is_refused(ctx, new):
    # with large pages its table is short, but its positions pass 32 bits
    s = Server(2, 4096, 4000, page=2 ** 20)
    s.step([0, 2 ** 31 - 8], [3, 5])
    got, *_ = s.build([7, ctx], [1, new], capacity=5000, rows=64)
    assert int(s.status[0]) == 1 << kap.ERR_CAPACITY
    assert not got["bt_indptr"].any() and not got["new_indptr"].any() and (got["slot"] == -9).all()
    s.expect_state()
