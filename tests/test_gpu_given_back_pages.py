"""Pages that a request has given back itself (a sliding window's past): negative entries of the page table.  kap_release_pages puts only pages on the
stack, kap_build_block_tables reports new rows that would lie on no page.  Everything is a whole number and has to be equal."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap
from test_gpu_block_tables import Server

pytestmark = pytest.mark.gpu
INDEX, FULL = 1 << kap.ERR_DEVICE_INDEX, 1 << kap.ERR_CAPACITY


def _give_back(s, dead):
    """what a program does with pages that no row sees any more: (request, logical page) pairs; onto the stack, and out of the table"""
    for r, i in dead:
        s.free[s.count] = s.table[r, i]
        s.count += 1
        s.table[r, i] = -1 - (r + i) % 5                           # any negative number
    for name, a in (("page_table", s.table), ("free_pages", s.free), ("free_count", [s.count])):
        s.dev[name].copy_(gu.i32(a))


def _released(s, request, keep=None):
    """the rules of a release on the host's copy"""
    moved = []
    for i, r in enumerate(request):
        left = min(s.held[r], 0 if keep is None else (keep[i] + s.page - 1) // s.page)
        moved += [p for p in s.table[r, left:s.held[r]] if p >= 0]
        s.held[r] = left
    s.free[s.count:s.count + len(moved)] = moved[::-1]
    s.count += len(moved)
    s.expect_state()


@pytest.mark.parametrize("batch,dead", [(1, 0.5), (5, 0.5), (40, 0.02), (40, 1.0), (300, 0.3), (1023, 0.5), (1025, 0.5), (2500, 0.1)])
def test_a_release_puts_pages_alone_on_the_stack(batch, dead):
    rng = np.random.default_rng(batch)
    s = Server(batch + 3, 40, 40 * batch + 50)
    request, ctx = rng.permutation(batch + 3)[:batch], np.zeros(batch, dtype=np.int64)
    for n_new in (rng.integers(0, 500, batch), rng.integers(0, 60, batch)):
        s.step(ctx, n_new, request)
        ctx += n_new
    # pages before the last 40 tokens, the first page apart
    _give_back(s, [(r, i) for r, c in zip(request, ctx) for i in range(1, max(1, (c - 40) // 16)) if rng.random() < dead])
    s.step(ctx, None, request)                                     # the given-back pages are taken again, by this request or another
    ctx += 1
    some, keep = request[:batch // 2 + 1], rng.integers(0, 300, batch // 2 + 1)
    s.release(some, keep)
    _released(s, some, keep)
    s.release()
    _released(s, range(len(s.held)))
    assert int(s.status[0]) == 0
    assert sorted(s.free[:s.count]) == list(range(len(s.free)))    # every page once, and nothing else


def test_the_stack_needs_room_for_pages_alone():
    s = Server(2, 12, 20)
    s.step([0, 0], [100, 60])                                      # 7 and 4 pages
    _give_back(s, [(0, 1), (0, 2), (1, 0)])
    # the eight pages that are left fit into a stack of exactly their number
    exact = dict(s.dev, free_pages=s.dev["free_pages"][:s.count + 8].clone())
    for room, status in ((7, FULL), (8, 0)):
        state = dict(exact, free_pages=exact["free_pages"][:s.count + room].clone(), pages_held=s.dev["pages_held"].clone(), free_count=s.dev["free_count"].clone())
        s.status.zero_()
        kap.release_pages(None, **state, device_status=s.status)
        assert int(s.status[0]) == status
        assert state["pages_held"].tolist() == ([7, 4] if status else [0, 0]) and int(state["free_count"][0]) == s.count + (0 if status else 8)
        if status:
            assert torch.equal(state["free_pages"][:s.count], exact["free_pages"][:s.count])
    assert torch.equal(state["free_pages"].sort().values.cpu(), torch.arange(20, dtype=torch.int32))


@pytest.mark.parametrize("batch", [3, 1200])
def test_new_rows_need_a_page(batch):
    s = Server(batch, 12, 20 + 2 * batch)
    tail = [20] * (batch - 3)
    s.step([70, 40, 5] + tail)                                     # 5, 3 and 1 pages
    _give_back(s, [(0, 0), (0, 1), (0, 2), (1, 2)])
    for ctx, new, status in (([71, 20, 6], [1, 5, 1], 0),          # on pages that are there
                             ([71, 40, 6], [1, 1, 1], INDEX),      # a row on logical page 2 of request 1
                             ([71, 20, 6], [1, 20, 1], INDEX),     # the last rows of a chunk
                             ([71, 48, 6], [1, 3, 1], 0),          # behind it: a page of its own
                             ([47, 48, 6], [1, 3, 1], INDEX), ([47, 48, 6], [0, 3, 1], 0),     # without rows nothing is needed
                             ([0, 48, 6], [100, 3, 1], INDEX)):
        s.status.zero_()
        state = {k: v.clone() for k, v in s.dev.items()}
        got, *rest = s.build(ctx + tail, new + [1] * len(tail))
        assert int(s.status[0]) == status
        if status:
            assert not got["bt_indptr"].any() and not got["new_indptr"].any()
            assert all(torch.equal(s.dev[k], state[k]) for k in state)
        else:
            s.expect_build(got, ctx + tail, *rest)


def test_long_chunks_on_pages_held():
    # every place of a chunk's pages, of several chunks in one step
    s = Server(40, 500, 19000)                                     # 18073 pages are needed
    ctx, new = np.arange(40) * 37, np.full(40, 6500)
    s.step(ctx, new)                                               # more than 400 pages each
    s.step(ctx, new)                                               # the same rows again: nothing is taken
    for r, i in ((0, 0), (1, 2), (7, 1 + (7 * 37) // 16), (7, 34), (7, 200), (33, 300), (39, 400), (39, 496), (38, 493)):
        was, held = int(s.table[r, i]), bool(i < s.held[r])
        s.table[r, i] = -1
        s.dev["page_table"].copy_(gu.i32(s.table))
        s.status.zero_()
        needed = ctx[r] // 16 <= i < (ctx[r] + 6500 + 15) // 16
        got, *rest = s.build(ctx, new)
        assert held and int(s.status[0]) == (INDEX if needed else 0)
        if not needed:
            s.expect_build(got, ctx, *rest)
        s.expect_state()
        s.table[r, i] = was
        s.dev["page_table"].copy_(gu.i32(s.table))
    s.status.zero_()
    s.step(ctx, new)


def test_an_index_beyond_the_row_is_not_followed():
    # the look-up of the first row's page stays inside the table; such a step is refused
    s = Server(3, 12, 40)
    s.step([10, 10, 10])
    for ctx in (12 * 16, 10 ** 6, 2 ** 31 - 2):
        s.status.zero_()
        got, *_ = s.build([11, 11, ctx], capacity=60)
        assert int(s.status[0]) == FULL and not got["bt_indptr"].any()
        s.expect_state()


def test_a_captured_release_meets_both():
    s = Server(4, 12, 60)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kap.release_pages(None, **s.dev, device_status=s.status)
    for dead in ([], [(0, 1), (2, 0), (2, 1)], []):
        s.step([0, 0, 0, 0], [50, 0, 60, 170])
        _give_back(s, dead)
        graph.replay()
        torch.cuda.synchronize()
        _released(s, range(4))
        assert int(s.status[0]) == 0 and sorted(s.free[:s.count]) == list(range(60))


def test_windowed_requests_that_give_their_past_back():
    """a server whose layers all look through a window of 100 tokens: the past goes back as it falls out of every later row's sight, results stay those of
    the whole cache, and in the end every page is on the stack once"""
    window, hq, hkv, d, steps = 100, 8, 2, 128, [(150, 90), (40, 1), (1, 1), (1, 130), (70, 1), (1, 1)]
    g = torch.Generator(device=gu.DEV).manual_seed(3)
    rand = lambda *sh: torch.randn(sh, device=gu.DEV, generator=g).to(torch.bfloat16)      # noqa: E731
    s = Server(2, 40, 24)
    pool = torch.full((24, 2, hkv, 16, d), float("nan"), dtype=torch.bfloat16, device=gu.DEV)
    ws = kap.Workspace(max_items=kap.chunk_attn_items(), max_rows_per_item=64, max_batch=2)
    ctx, plain = np.zeros(2, dtype=np.int64), [[None, None], [None, None]]
    for new in steps:
        new = np.array(new)
        got, pages, n, req = s.build(ctx, new)
        assert int(s.status[0]) == 0
        s.expect_build(got, ctx, pages, n, req)
        rows = int(new.sum())
        q, k, v = rand(rows, hq, d), rand(rows, hkv, d), rand(rows, hkv, d)
        tables = gu.i32(got["bt_indptr"]), gu.i32(got["bt_pages"])
        kap.append_kv(k, v, pool, *tables, gu.i32(ctx), new_indptr=gu.i32(got["new_indptr"]))
        out = torch.full_like(q, float("nan"))
        kap.chunk_attn(q, gu.i32(got["new_indptr"]), pool, *tables, gu.i32(ctx + new), out, ws, window=window)
        ws.check()
        at = 0
        for b in range(2):
            x = slice(at, at + int(new[b]))
            at += int(new[b])
            plain[b] = [new_part.double() if old is None else torch.cat([old, new_part.double()]) for old, new_part in zip(plain[b], (k[x], v[x]))]
            keys, values = (t.repeat_interleave(hq // hkv, 1) for t in plain[b])
            pos, t = torch.arange(ctx[b], ctx[b] + new[b], device=gu.DEV)[:, None], torch.arange(len(keys), device=gu.DEV)[None]
            z = torch.einsum("nhd,thd->hnt", q[x].double(), keys) * d ** -0.5
            w = torch.softmax(torch.where((t <= pos) & (t > pos - window), z, -torch.inf), -1)
            ref, size = torch.einsum("hnt,thd->nhd", w, values), torch.einsum("hnt,thd->nhd", w, values.abs())
            # weights and results are rounded to bf16; scores of fp32 (as for the calls' own tests)
            assert bool(((out[x].double() - ref).abs() <= 2.0 ** -8 * (size + ref.abs()) + 1e-3 * size).all())
        ctx += new
        # what the next row does not see: tokens up to ctx - window
        dead = [(b, i) for b in range(2) for i in range(int(ctx[b] - window + 1) // 16) if s.table[b, i] >= 0]
        for b, i in dead:
            pool[int(s.table[b, i])] = float("nan")
        _give_back(s, dead)
    s.release()
    _released(s, range(2))
    assert int(s.status[0]) == 0 and sorted(s.free[:s.count]) == list(range(24))
