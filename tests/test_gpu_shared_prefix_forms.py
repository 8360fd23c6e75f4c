"""kap_shared_prefix_attn in forms that test_gpu_shared_prefix.py leaves out: head groups of 1, 2 and 16 on the tensor-memory kernel,
launches without programmatic ordering, and inputs written by the kernels directly in front of the call.  Tolerances as there."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap
from test_gpu_shared_prefix import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", [kap.KV_HND, kap.KV_NHD])
@pytest.mark.parametrize("members", [40, 129, 300])
@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (4, 2), (16, 8), (16, 1)])
def test_head_groups_of_every_size_over_many_rows(hq, hkv, members, layout):
    # 40 query rows a KV head (one tile, partly filled) to 4800 (19 blocks of two tiles); a second group with a prefix of its own
    rng = np.random.default_rng(members + hq)
    if hq // hkv == 1 and members == 300:
        layout = kap.KV_HND if hq == 1 else kap.KV_NHD
    Case(40 + members, [(83, [(1, int(t)) for t in rng.integers(1, 40, members)]), (7, [(2, 2), (1, 33), (3, 70)] * 12)], hq, hkv, layout).check()


@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 4)])
def test_windows_of_small_head_groups_that_reach_into_the_prefix(hq, hkv):
    Case(41, [(11, [(6, 2), (1, 0), (3, 1), (16, 20)] * 9)], hq, hkv).check()


@pytest.fixture
def ordinary_launches():
    kap.set_launch_options(use_pdl=0)
    yield
    kap.set_launch_options(use_pdl=1)


GROUPS = [(150, [(2, 40 + i) for i in range(24)]), (3, [(1, 9), (4, 300)]), (0, [(2, 50)]), (40, [(1, 0)] * 40)]


def test_the_same_results_without_programmatic_launches(ordinary_launches):
    c = Case(42, GROUPS)
    ordinary = c.check()
    kap.set_launch_options(use_pdl=1)
    again = c.call()
    assert torch.equal(ordinary[0], again[0]) and torch.equal(ordinary[1], again[1])


@pytest.mark.parametrize("pdl", [0, 1])
def test_inputs_written_just_before_the_call(pdl):
    # queries, contexts and the pool change between calls that follow one another without a pause, in a stream and in a graph
    c = Case(43, [(200, [(1, 30 + i) for i in range(33)]), (20, [(4, 80), (4, 17)])], 32, 8, poison=0.0)
    qs = [c.q.clone(), (c.q.float() * -0.7).to(torch.bfloat16)]
    ctxs = [gu.i32(c.ctx), gu.i32(np.maximum(c.ctx - 7, 4))]
    pools = [c.pool.clone(), c.pool.roll(1, 0)]
    c.ws = c.workspace()
    q, qi, pool, bti, btp, ctx = c.arrays()

    def step(i, out):
        q.copy_(qs[i])
        pool.copy_(pools[i])
        ctx.copy_(ctxs[i])
        kap.shared_prefix_attn(q, qi, pool, bti, btp, ctx, out, c.ws)

    try:
        kap.set_launch_options(use_pdl=pdl)
        want = []
        for i in (0, 1):
            want.append(torch.empty_like(c.q))
            q.copy_(qs[i])
            pool.copy_(pools[i])
            ctx.copy_(ctxs[i])
            torch.cuda.synchronize()
            kap.shared_prefix_attn(q, qi, pool, bti, btp, ctx, want[i], c.ws)
            torch.cuda.synchronize()
        assert not torch.equal(want[0], want[1])
        got = [torch.empty_like(c.q) for _ in range(40)]
        for n, out in enumerate(got):
            step(n % 2, out)
        for n, out in enumerate(got):
            assert torch.equal(out, want[n % 2]), f"call {n}"
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for n in range(6):
                step(n % 2, got[n])
        for _ in range(5):
            for out in got[:6]:
                out.zero_()
            graph.replay()
            torch.cuda.synchronize()
            for n in range(6):
                assert torch.equal(got[n], want[n % 2]), f"captured call {n}"
        c.ws.check()
    finally:
        kap.set_launch_options(use_pdl=1)
