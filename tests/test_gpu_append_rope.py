"""kap_append_kv_rope on the GPU against a 64-bit rotation on the host.

Tolerance: a result is one rounding to bf16 (at most 2^-8 of the value) of a fp32 value a c - b s.  c and s carry the
rounding of the reduced angle (at most pi 2^-24) and sincospif's error (2 ulp, 2^-23): together below 2^-21; the products and
the sum add 3 roundings of 2^-24 of at most |a| + |b|: 2^-21 in all.  A position of 10^9 rounds its 64-bit angle by up to
2^-54 10^9 rad four times (the product here and there, the turns, the constant), below 2^-21: 2^-20 covers both."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap, synth

pytestmark = pytest.mark.gpu
D, PAGE = 128, 16


def _rotated(x, angle, rot, interleaved):
    """x f64 [rows, heads, D], angle f64 [rows, rot / 2]; returns (result, |a| + |b|)"""
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    c, s = np.cos(angle)[:, None, :], np.sin(angle)[:, None, :]
    y, size = x.copy(), np.abs(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size


def _near(got, ref, size):
    bad = np.abs(got - ref) > 2.0 ** -8 * np.abs(ref) + 2.0 ** -20 * size
    assert not bad.any(), f"{bad.sum()} values off, worst {np.abs(got - ref)[bad].max()}"


class Case:
    def __init__(self, seed, n_new, ctx, hq=8, hkv=2, rot=128, interleaved=False, layout=kap.KV_HND, fused=False, one=False, base=500000.0):
        rng = np.random.default_rng(seed)
        self.n_new, self.ctx, self.hq, self.hkv, self.rot, self.inter, self.layout = np.asarray(n_new), np.asarray(ctx), hq, hkv, rot, interleaved, layout
        self.rows = int(self.n_new.sum())
        self.indptr = np.concatenate([[0], np.cumsum(self.n_new)]).astype(np.int32)
        pages = (self.ctx + self.n_new + PAGE - 1) // PAGE
        self.bt_indptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
        self.n_pages = min(int(pages.sum()), 64) + 3
        # the pages behind the window may repeat (nobody writes there); those of the window are the sequence's own
        self.bt = rng.integers(0, 3, int(pages.sum())).astype(np.int32)
        fresh = iter(rng.permutation(self.n_pages - 3) + 3)
        for b in range(len(pages)):
            for lp in range(int(self.ctx[b]) // PAGE, int(pages[b])):
                self.bt[self.bt_indptr[b] + lp] = next(fresh)
        self.inv = (base ** (-np.arange(rot // 2) / (rot // 2))).astype(np.float32)
        self.qkv = synth.normal_bf16((self.rows, hq + 2 * hkv, D), 1.0, rng)
        shape = (self.n_pages, 2, hkv, PAGE, D) if layout == kap.KV_HND else (self.n_pages, 2, PAGE, hkv, D)
        self.pool = synth.normal_bf16(shape, 0.5, rng)
        dev = gu.bits_to_dev(self.qkv)
        parts = dev[:, :hq], dev[:, hq:hq + hkv], dev[:, hq + hkv:]
        self.q, self.k, self.v = parts if fused else [x.contiguous() for x in parts]
        self.d_pool, self.d_ctx = gu.bits_to_dev(self.pool), gu.i32(self.ctx)
        self.status = torch.zeros(1, dtype=torch.int32, device=gu.DEV)
        self.d_indptr = None if one else gu.i32(self.indptr)
        self.d_bt = gu.i32(self.bt_indptr), gu.i32(self.bt)

    def call(self, **kw):
        a = dict(q_out=None if self.q is None else torch.zeros_like(self.q), new_indptr=self.d_indptr, interleaved=self.inter, kv_layout=self.layout,
                 device_status=self.status)
        a.update(kw)
        kap.append_kv_rope(self.q, self.k, self.v, self.d_pool, *self.d_bt, self.d_ctx, torch.from_numpy(self.inv).to(gu.DEV), **a)
        return a["q_out"]

    def check(self, q_out, positions=None, freq_axis=None, offset=None, advanced=True):
        """positions int [axes, rows]"""
        torch.cuda.synchronize()
        place = np.concatenate([self.ctx[b] + np.arange(n) for b, n in enumerate(self.n_new)])
        seq = np.repeat(np.arange(len(self.n_new)), self.n_new)
        if positions is None:
            pos = (place + (0 if offset is None else offset[seq]))[:, None].astype(np.float64)
        else:
            pos = positions.T[:, np.zeros(self.rot // 2, dtype=int) if freq_axis is None else freq_axis].astype(np.float64)
        angle = pos * self.inv.astype(np.float64)
        x = synth.bf16_bits_to_f64(self.qkv)
        q, q_size = _rotated(x[:, :self.hq], angle, self.rot, self.inter)
        k, k_size = _rotated(x[:, self.hq:self.hq + self.hkv], angle, self.rot, self.inter)
        _near(gu.dev_bf16_to_f64(q_out), q, q_size)
        heads_first = (lambda p: p) if self.layout == kap.KV_HND else (lambda p: p.transpose(0, 1, 3, 2, 4))
        got, was = heads_first(gu.dev_to_bits(self.d_pool)), heads_first(self.pool).copy()
        page = self.bt[self.bt_indptr[seq] + place // PAGE]
        slot = place % PAGE
        _near(synth.bf16_bits_to_f64(np.ascontiguousarray(got[page, 0, :, slot])), k, k_size)
        np.testing.assert_array_equal(got[page, 1, :, slot], self.qkv[:, self.hq + self.hkv:])
        was[page, :, :, slot] = got[page, :, :, slot]
        np.testing.assert_array_equal(got, was, err_msg="a slot that belongs to no new token was written")
        if self.rot < D:                                                         # the rest of the head is copied bit for bit
            np.testing.assert_array_equal(gu.dev_to_bits(q_out)[..., self.rot:], self.qkv[:, :self.hq, self.rot:])
        np.testing.assert_array_equal(self.d_ctx.cpu().numpy(), self.ctx + (self.n_new if advanced else 0))
        assert int(self.status.item()) == 0


@pytest.mark.parametrize("layout", [kap.KV_HND, kap.KV_NHD])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [16, 48, 64, 128])
def test_one_token_per_sequence(rot, interleaved, layout):
    c = Case(1, [1] * 5, [0, 15, 16, 1000, 131071], rot=rot, interleaved=interleaved, layout=layout, fused=True, one=True)
    c.check(c.call())


@pytest.mark.parametrize("hq,hkv", [(1, 1), (32, 8), (16, 1), (6, 6)])
def test_head_counts(hq, hkv):
    c = Case(2, [3, 0, 1, 40], [7, 0, 31, 0], hq=hq, hkv=hkv)
    c.check(c.call())


@pytest.mark.parametrize("n_new,ctx", [([1], [0]), ([17], [15]), ([0, 0, 5], [3, 4, 5]), ([5, 0, 0], [3, 4, 5]), ([200, 1, 33], [131000, 9, 64])])
def test_windows(n_new, ctx):
    c = Case(3, n_new, ctx, interleaved=True, fused=True)
    c.check(c.call())
    c = Case(3, n_new, ctx, layout=kap.KV_NHD)
    c.check(c.call(advance=False), advanced=False)


@pytest.mark.parametrize("far", [0, 999_983, 16_777_217, 1_000_000_007])
def test_far_positions_and_several_axes(far):
    c = Case(4, [9, 30], [40, 0], rot=96)
    rng = np.random.default_rng(far % 1000)
    pos = rng.integers(0, 40, (3, c.rows)).astype(np.int32)
    pos[0] += far
    axis = rng.integers(0, 3, 48).astype(np.uint8)
    wide = torch.zeros((3, c.rows + 5), dtype=torch.int32, device=gu.DEV)        # rows of positions with padding behind them
    wide[:, :c.rows] = gu.i32(pos)
    c.check(c.call(positions=wide[:, :c.rows], freq_axis=axis), positions=pos, freq_axis=axis)
    one = Case(4, [9, 30], [40, 0], rot=96)
    one.check(one.call(positions=gu.i32(pos[0])), positions=pos[:1])


def test_position_offset():
    c = Case(5, [2, 7, 1], [30, 5, 100])
    offset = np.array([-12, 0, 4321], dtype=np.int32)
    c.check(c.call(position_offset=gu.i32(offset)), offset=offset)


def test_in_place_equals_out_of_place_and_kv_only():
    a, b, c = (Case(6, [4, 9], [3, 70], fused=f) for f in (False, True, False))
    out = a.call()
    b.call(q_out=b.q)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(gu.dev_to_bits(b.q), gu.dev_to_bits(out))
    np.testing.assert_array_equal(gu.dev_to_bits(b.d_pool), gu.dev_to_bits(a.d_pool))
    c.q = None
    c.call(q_out=None)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(gu.dev_to_bits(c.d_pool), gu.dev_to_bits(a.d_pool))


def test_rows_of_nobody_are_left_alone():
    c = Case(7, [3, 4], [10, 20])
    c.d_indptr = gu.i32([2, 4, 6])                                               # rows 0, 1 and 6 belong to no sequence
    before = gu.dev_to_bits(c.d_pool)
    out = torch.full_like(c.q, 7.0)
    c.call(q_out=out)
    torch.cuda.synchronize()
    rows = gu.dev_bf16_to_f64(out)
    assert (rows[[0, 1, 6]] == 7.0).all() and (rows[2:6] != 7.0).any(axis=(1, 2)).all()
    changed = (gu.dev_to_bits(c.d_pool) != before).any(axis=(2, 4))              # [page, k/v, slot]
    assert changed.sum() == 4 * 2


def test_bad_pages_are_reported_and_nothing_is_written():
    for bad in (-1, 10 ** 6):
        c = Case(8, [3, 2], [0, 0])
        c.bt[0] = bad
        c.d_bt = gu.i32(c.bt_indptr), gu.i32(c.bt)
        before = c.pool.copy()
        c.call()
        torch.cuda.synchronize()
        assert int(c.status.item()) == 1 << kap.ERR_DEVICE_INDEX
        after = gu.dev_to_bits(c.d_pool)
        page = c.bt[c.bt_indptr[1]]
        before[page, :, :, :2] = after[page, :, :, :2]
        np.testing.assert_array_equal(after, before)
    c = Case(8, [3, 2], [0, 0])
    c.d_ctx = gu.i32([-4, 0])
    c.call(device_status=None)                                                   # without a status word: not written, not reported
    torch.cuda.synchronize()
    page = c.bt[0]
    np.testing.assert_array_equal(gu.dev_to_bits(c.d_pool)[page], c.pool[page])


def test_the_window_past_the_block_table():
    c = Case(9, [20], [0])
    c.d_bt = gu.i32([0, 1]), gu.i32(c.bt)                                        # one page only: tokens 16 .. 19 have none
    c.call()
    torch.cuda.synchronize()
    assert int(c.status.item()) == 1 << kap.ERR_DEVICE_INDEX
    after = gu.dev_to_bits(c.d_pool)
    assert (after[c.bt[1]] == c.pool[c.bt[1]]).all() and (after[c.bt[0]] != c.pool[c.bt[0]]).any()


def test_binding_refuses_what_it_cannot_pass_on():
    c = Case(10, [2], [0])
    for change in (dict(q_out=c.q.float()), dict(positions=torch.zeros(3, dtype=torch.int32, device=gu.DEV)), dict(freq_axis=[0] * 3),
                   dict(positions=torch.zeros(2, dtype=torch.int64, device=gu.DEV))):
        with pytest.raises(kap.KapError):
            c.call(**change)
    c.q = c.q.transpose(1, 2).contiguous().transpose(1, 2)                       # heads not contiguous
    with pytest.raises(kap.KapError):
        c.call(q_out=torch.zeros_like(c.k))
