"""kap_append_kv_norm_rope on the GPU against norms and rotation in 64 bits on the host.

Tolerance: as for kap_append_kv_rope, one rounding to bf16 (2^-8 of the value) of a fp32 value, the rotation's part of which is within 2^-20 of
|a| + |b|.  The norm adds: the sum of 128 squares (17 roundings in a row at most, 2^-24 each, halved by the root), rsqrt (2 ulp, 2^-22), the products
with the weight and with 1 / 128 (3 roundings): below 2^-19 of each of a and b.  2^-18 (|a| + |b|) covers both."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap, synth
from test_gpu_append_rope import Case, _rotated

pytestmark = pytest.mark.gpu
D, PAGE = 128, 16


def _near(got, ref, size):
    bad = np.abs(got - ref) > 2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * size
    assert not bad.any(), f"{bad.sum()} values off, worst {np.abs(got - ref)[bad].max()}"


class Normed(Case):
    def __init__(self, *a, weights="shared", dtype=torch.bfloat16, unit=False, eps=1e-6, **kw):
        super().__init__(*a, **kw)
        g = torch.Generator(device=gu.DEV).manual_seed(99)
        shape = lambda heads: (heads, D) if weights == "per head" else (D,)         # noqa: E731
        make = lambda heads: None if weights is None else (torch.randn(shape(heads), device=gu.DEV, generator=g) + (0.0 if unit else 1.0)).to(dtype)   # noqa: E731
        self.qw, self.kw, self.unit, self.eps = make(self.hq), make(self.hkv), unit, eps

    def call(self, **kw):
        a = dict(q_out=None if self.q is None else torch.zeros_like(self.q), new_indptr=self.d_indptr, interleaved=self.inter, kv_layout=self.layout,
                 device_status=self.status, q_weight=self.qw, k_weight=self.kw, unit_offset=self.unit, eps=self.eps)
        a.update(kw)
        kap.append_kv_norm_rope(self.q, self.k, self.v, self.d_pool, *self.d_bt, self.d_ctx, torch.from_numpy(self.inv).to(gu.DEV), **a)
        return a["q_out"]

    def normed(self, x, w):
        w = 1.0 if w is None else w.double().cpu().numpy() + (1.0 if self.unit else 0.0)
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + self.eps) * w

    def check(self, q_out):
        torch.cuda.synchronize()
        place = np.concatenate([self.ctx[b] + np.arange(n) for b, n in enumerate(self.n_new)])
        seq = np.repeat(np.arange(len(self.n_new)), self.n_new)
        angle = place[:, None] * self.inv.astype(np.float64)
        x = synth.bf16_bits_to_f64(self.qkv)
        q, q_size = _rotated(self.normed(x[:, :self.hq], self.qw), angle, self.rot, self.inter)
        k, k_size = _rotated(self.normed(x[:, self.hq:self.hq + self.hkv], self.kw), angle, self.rot, self.inter)
        if q_out is not None:
            _near(gu.dev_bf16_to_f64(q_out), q, q_size)
        got = gu.dev_to_bits(self.d_pool)
        want = self.pool.copy()
        page = self.bt[self.bt_indptr[seq] + place // PAGE]
        heads = got.transpose(0, 1, 3, 2, 4) if self.layout == kap.KV_NHD else got
        was = want.transpose(0, 1, 3, 2, 4) if self.layout == kap.KV_NHD else want
        _near(synth.bf16_bits_to_f64(np.ascontiguousarray(heads[page, 0, :, place % PAGE])), k, k_size)
        was[page, 1, :, place % PAGE] = self.qkv[:, self.hq + self.hkv:]
        was[page, 0, :, place % PAGE] = heads[page, 0, :, place % PAGE]
        assert np.array_equal(got, want), "v, or something beyond the rows' slots"
        assert int(self.status[0]) == 0


@pytest.mark.parametrize("weights", ["shared", "per head", None])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("layout", [kap.KV_HND, kap.KV_NHD])
def test_forms(weights, dtype, interleaved, layout):
    c = Normed(1, [3, 0, 20, 1], [5, 7, 100, 0], interleaved=interleaved, layout=layout, weights=weights, dtype=dtype, fused=interleaved)
    c.check(c.call())


@pytest.mark.parametrize("rot", [16, 48, 64, 112, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_partly_rotated_heads(rot, interleaved):
    c = Normed(2, [9, 4], [33, 131000], rot=rot, interleaved=interleaved)
    c.check(c.call())


@pytest.mark.parametrize("hq,hkv", [(1, 1), (3, 3), (32, 8), (5, 1), (64, 4)])
def test_head_counts(hq, hkv):
    c = Normed(3, [2, 17], [1, 15], hq=hq, hkv=hkv, weights="per head")
    c.check(c.call())


def test_weights_around_zero():
    c = Normed(4, [5, 2], [1, 15], unit=True)
    c.check(c.call())
    c = Normed(4, [5, 2], [1, 15], unit=True, weights="per head", dtype=torch.float32, eps=0.5)
    c.check(c.call())


def test_small_and_large_heads():
    for scale in (1e-20, 1e-3, 1e15):
        c = Normed(5, [6], [40], eps=1e-6 if scale > 1e-10 else 0.0 if scale == 1e-3 else 1e-6)
        for t in (c.q, c.k):
            t.copy_(t.float() * scale)
        bits = np.concatenate([gu.dev_to_bits(c.q), gu.dev_to_bits(c.k)], 1)
        c.qkv[:, :c.hq + c.hkv] = bits
        c.check(c.call())


def test_a_head_of_zeros_stays_zero():
    c = Normed(6, [3], [10])
    c.q.zero_(), c.k.zero_()
    c.qkv[:, :c.hq + c.hkv] = 0
    q_out = c.call()
    assert bool((q_out == 0).all())
    c.check(q_out)


def test_a_nan_stays_in_its_head():
    c = Normed(7, [3], [10])
    c.q[1, 2, 5] = float("nan")
    q_out = c.call()
    torch.cuda.synchronize()
    nan = q_out.isnan().any(-1)
    assert bool(nan[1, 2]) and int(nan.sum()) == 1


def test_single_tokens_in_place_and_advance():
    c = Normed(8, [1] * 9, list(range(9)), one=True)
    before = c.q.clone()
    c.call(q_out=c.q, advance=True)
    c.check(c.q)
    assert c.d_ctx.tolist() == list(range(1, 10)) and not torch.equal(before, c.q)
    c = Normed(9, [4, 2], [3, 8])
    c.call(advance=True)
    assert c.d_ctx.tolist() == [7, 10]


def test_k_and_v_alone():
    c = Normed(10, [4, 2], [3, 8])
    c.q, c.qw = None, None
    c.call()
    c.check(None)


def test_a_captured_call_repeats():
    c = Normed(11, [7, 30], [3, 40], weights="per head")
    first = c.call(advance=False)
    out = torch.zeros_like(c.q)
    inv = torch.from_numpy(c.inv).to(gu.DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kap.append_kv_norm_rope(c.q, c.k, c.v, c.d_pool, *c.d_bt, c.d_ctx, inv, q_out=out, new_indptr=c.d_indptr, q_weight=c.qw, k_weight=c.kw, advance=False)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, out)
    c.check(out)


def test_without_norms_the_rotation_alone_is_as_before():
    # unit norms: heads that are normalised already come out as append_kv_rope leaves them, to a rounding of the norm
    c = Normed(12, [5], [9], weights=None, eps=0.0)
    sign = torch.where(torch.rand(c.q.shape, device=gu.DEV) < 0.5, -1.0, 1.0).to(torch.bfloat16)
    c.q.copy_(sign)
    got = c.call(advance=False)
    ref = torch.zeros_like(got)
    kap.append_kv_rope(c.q, c.k, c.v, c.d_pool, *c.d_bt, c.d_ctx, torch.from_numpy(c.inv).to(gu.DEV), q_out=ref, new_indptr=c.d_indptr, advance=False)
    assert float((got.double() - ref.double()).abs().max()) <= 2.0 ** -7


def test_refusals():
    c = Normed(13, [5], [9])
    for kw in (dict(q_weight=c.qw.half()), dict(q_weight=c.qw[:64]), dict(q_weight=c.qw.float()), dict(k_weight=torch.ones(3, D, device=gu.DEV, dtype=torch.bfloat16)),
               dict(q_weight=c.qw.cpu()), dict(eps=-1.0), dict(eps=float("nan")), dict(q_weight=torch.ones(129, device=gu.DEV, dtype=torch.bfloat16)[1:])):
        with pytest.raises(kap.KapError) as e:
            c.call(**kw)
        assert e.value.code == kap.ERR_INVALID_ARG
