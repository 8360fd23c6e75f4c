"""Forms of a mixed step's calls: kap_append_kv_norm_rope with given positions, several axes and offsets, kap_chunk_attn and kap_build_block_tables as
ordinary launches, kap_build_block_tables without its optional arrays."""
import numpy as np
import pytest
import torch

import gpu_util as gu
import test_gpu_chunk_attn as chunk
from paper_2607_24260_b200 import kap, synth
from test_gpu_append_norm import Normed, _near
from test_gpu_append_rope import _rotated
from test_gpu_block_tables import Server

pytestmark = pytest.mark.gpu
D, PAGE = 128, 16


class Placed(Normed):
    def check_at(self, q_out, pos):
        """pos f64 [rows, rotated pairs]; tolerances as for the norm append's other tests"""
        torch.cuda.synchronize()
        angle = pos * self.inv.astype(np.float64)
        x = synth.bf16_bits_to_f64(self.qkv)
        q, q_size = _rotated(self.normed(x[:, :self.hq], self.qw), angle, self.rot, self.inter)
        k, k_size = _rotated(self.normed(x[:, self.hq:self.hq + self.hkv], self.kw), angle, self.rot, self.inter)
        _near(gu.dev_bf16_to_f64(q_out), q, q_size)
        seq = np.repeat(np.arange(len(self.n_new)), self.n_new)
        place = np.concatenate([self.ctx[b] + np.arange(n) for b, n in enumerate(self.n_new)])
        heads = gu.dev_to_bits(self.d_pool)
        heads = heads.transpose(0, 1, 3, 2, 4) if self.layout == kap.KV_NHD else heads
        page = self.bt[self.bt_indptr[seq] + place // PAGE]           # rows lie at their logical index, whatever their position
        _near(synth.bf16_bits_to_f64(np.ascontiguousarray(heads[page, 0, :, place % PAGE])), k, k_size)
        assert np.array_equal(heads[page, 1, :, place % PAGE], self.qkv[:, self.hq + self.hkv:])
        assert int(self.status[0]) == 0


@pytest.mark.parametrize("interleaved,layout", [(False, kap.KV_HND), (True, kap.KV_NHD)])
@pytest.mark.parametrize("weights", ["shared", "per head", None])
def test_norms_with_given_positions(weights, interleaved, layout):
    c = Placed(21, [3, 0, 20, 1], [5, 7, 100, 0], interleaved=interleaved, layout=layout, weights=weights)
    pos = np.random.default_rng(1).integers(0, 200000, c.rows).astype(np.int32)
    c.check_at(c.call(positions=gu.i32(pos)), np.repeat(pos[:, None].astype(np.float64), c.rot // 2, 1))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot,axes", [(128, 3), (64, 2), (48, 4)])
def test_norms_with_several_axes(rot, axes, interleaved):
    c = Placed(22, [9, 4, 1], [33, 1000, 0], rot=rot, interleaved=interleaved, fused=True)
    rng = np.random.default_rng(2)
    pos = rng.integers(0, 100000, (axes, c.rows)).astype(np.int32)
    axis = rng.integers(0, axes, rot // 2)
    c.check_at(c.call(positions=gu.i32(pos), freq_axis=axis.tolist()), pos.T[:, axis].astype(np.float64))


@pytest.mark.parametrize("one", [False, True])
def test_norms_with_an_offset_for_each_sequence(one):
    n = [1] * 5 if one else [3, 0, 17, 1, 2]
    c = Placed(23, n, [5, 7, 100, 0, 31], one=one)
    offset = np.array([0, 3, -5, 100000, 7], dtype=np.int32)
    seq = np.repeat(np.arange(5), n)
    place = np.concatenate([c.ctx[b] + np.arange(x) for b, x in enumerate(n)])
    c.check_at(c.call(position_offset=gu.i32(offset)), np.repeat((place + offset[seq])[:, None].astype(np.float64), c.rot // 2, 1))


def test_ordinary_launches_give_the_same_results():
    c = chunk.Case(24, chunk.MIXED, 8, 2)
    long = chunk.Case(25, [(1500, 12777)], 32, 8)
    want = [x.call() for x in (c, long)]
    s = Server(40, 40, 900)
    n_new = np.random.default_rng(3).integers(0, 90, 40)
    try:
        kap.set_launch_options(use_pdl=0)
        for x, (out, lse) in zip((c, long), want):
            got = x.call()
            assert torch.equal(out.nan_to_num(7.0), got[0].nan_to_num(7.0)) and torch.equal(lse.nan_to_num(7.0), got[1].nan_to_num(7.0))
        s.step(np.zeros(40, dtype=np.int64), n_new)
        s.step(n_new)
        s.release()
        s.expect_release()
    finally:
        kap.set_launch_options(use_pdl=1)


def test_tables_without_the_optional_arrays():
    s = Server(6, 10, 50)
    s.step([0, 16, 31, 5, 0, 0], [0, 3, 0, 0, 0, 0])                # request 1 holds two pages, 2 also two, 3 one
    held = s.held.copy()
    ip, pg = gu.i32([7] * 4), gu.i32([-9] * 8)
    kap.build_block_tables(gu.i32([1, 18, 40]), **s.dev, bt_indptr=ip, bt_pages=pg, device_status=s.status)
    assert list(held[:3]) == [0, 2, 2]
    first, third = s.free[s.count - 1], s.free[s.count - 2]          # request 0 takes the top, request 2 the next
    s.table[0, 0], s.table[2, 2], s.held[0], s.held[2] = first, third, 1, 3
    s.count -= 2
    assert ip.tolist() == [0, 1, 3, 6]
    assert pg.tolist() == [first, s.table[1, 0], s.table[1, 1], s.table[2, 0], s.table[2, 1], third, -9, -9]
    s.expect_state()
    assert int(s.status[0]) == 0


@pytest.mark.parametrize("norms", [False, True])
@pytest.mark.parametrize("indptr,length", [([0, 10, 4, 12], 0), ([0, 10, 4, 12], 3), ([0, 40, 1, 42], 0)])
def test_offsets_that_fall_write_nothing_in_front(indptr, length, norms):
    # rows that lie in front of their sequence's first one; the sequences' pages are in the middle of the pool, all others stay
    hq, hkv, rows, g = 8, 2, indptr[-1], torch.Generator(device=gu.DEV).manual_seed(30)
    rand = lambda heads: torch.randn((rows, heads, D), device=gu.DEV, generator=g).to(torch.bfloat16)      # noqa: E731
    q, k, v = rand(hq), rand(hkv), rand(hkv)
    pool = torch.full((40, 2, hkv, PAGE, D), 3.0, dtype=torch.bfloat16, device=gu.DEV)
    pages = np.arange(20, 29)                                       # three a sequence
    status = torch.zeros(1, dtype=torch.int32, device=gu.DEV)
    inv = torch.ones(D // 2, device=gu.DEV)
    call = kap.append_kv_norm_rope if norms else kap.append_kv_rope
    call(q, k, v, pool, gu.i32([0, 3, 6, 9]), gu.i32(pages), gu.i32([length] * 3), inv, q_out=torch.empty_like(q), new_indptr=gu.i32(indptr), advance=False, device_status=status)
    assert int(status[0]) == 1 << kap.ERR_DEVICE_INDEX
    keep = torch.ones(40, dtype=torch.bool, device=gu.DEV)
    keep[20:29] = False
    assert bool((pool[keep] == 3.0).all())
    # v of the rows that have an owner: those of the first sequence and of the last, whose first row is the offset's
    heads = pool.permute(0, 1, 3, 2, 4)
    for b, row in ((0, 0), (2, rows - 1)):
        pos = length + row - indptr[b]
        assert torch.equal(heads[20 + 3 * b + pos // PAGE, 1, pos % PAGE], v[row])
