"""kap_adjust_logits on the GPU against the rules in 64 bits.

Tolerance: the rules are at most four fp32 operations in a row (quotient or product, product f c, two differences, and the sums with the biases), each rounded by
2^-24 of its result; every intermediate result is at most |x| max(r, 1 / r) + f c + p + sum |bias|, so the fp32 value is within (6 + biases) 2^-24 of that; bf16
logits are rounded once more, by 2^-8 of the result."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


class Case:
    def __init__(self, seed, rows, vocab, dtype=F32, pad=0, out_pad=0, longest=200, biases=5, masks=None, spread=3.0, off=True):
        rng = np.random.default_rng(seed)
        self.rows, self.vocab, self.dtype = rows, vocab, dtype
        g = torch.Generator(device=gu.DEV).manual_seed(seed)
        self.logits = (torch.randn((rows, vocab + pad), device=gu.DEV, generator=g) * spread).to(dtype)[:, :vocab]
        self.out = torch.full((rows, vocab + out_pad), 7.0, dtype=dtype, device=gu.DEV)[:, :vocab]
        # words of which some come often, some outside the vocabulary
        self.history = np.minimum((vocab ** rng.random(rows * longest + 10)).astype(np.int64), vocab + 3).astype(np.int32)
        self.history[rng.integers(0, len(self.history), 5)] = -1
        n = rng.integers(0, longest + 1, (rows, 2))
        first = np.arange(rows) * longest
        ends = np.sort(n, 1)
        self.at = np.stack([first, first + ends[:, 0], first + ends[:, 1]], 1).astype(np.int64)
        pick = lambda off, *v: np.where(rng.random(rows) < 0.25, off, rng.choice(v, rows)).astype(np.float32)     # noqa: E731
        self.rep, self.pres, self.freq = pick(1.0, 1.3, 0.7, 2.0), pick(0.0, 0.6, -0.4), pick(0.0, 0.2, -0.1, 1.5)
        count = np.minimum(rng.integers(0, biases + 1, rows), vocab) if biases else np.zeros(rows, dtype=np.int64)
        self.bias_at = np.concatenate([[0], np.cumsum(count)]).astype(np.int32)
        self.bias_token = np.concatenate([np.sort(rng.integers(0, vocab, c)) for c in count] + [np.zeros(0, dtype=np.int64)]).astype(np.int32)
        self.bias_value = rng.normal(0, 5, len(self.bias_token)).astype(np.float32)
        self.masks = self.mask_row = None
        if masks:
            self.masks = rng.integers(-2 ** 31, 2 ** 31, (masks, (vocab + 31) // 32 + 1)).astype(np.int32)
            self.masks[:, ::3] = 0
            self.masks[:, 1::7] = -1
            self.mask_row = rng.integers(-1, masks, rows).astype(np.int32)
        self.status = torch.zeros(1, dtype=torch.int32, device=gu.DEV)

    def args(self, **drop):
        f = lambda a: torch.from_numpy(np.array(a)).to(gu.DEV)                     # noqa: E731
        a = dict(history=f(self.history), history_at=f(self.at), repetition=f(self.rep), presence=f(self.pres), frequency=f(self.freq),
                 bias_indptr=f(self.bias_at), bias_token=f(self.bias_token), bias_value=f(self.bias_value))
        if self.masks is not None:
            a.update(allowed=f(self.masks), allowed_row=f(self.mask_row))
        return a

    def expected(self, names):
        """(result, bound) in 64 bits, from the rules that `names` names"""
        x = self.logits.double().cpu().numpy()
        y, size = x.copy(), np.abs(x)
        for r in range(self.rows):
            b, a, e = self.at[r]
            inside = lambda t: t[(t >= 0) & (t < self.vocab)]                      # noqa: E731
            seen, said = np.zeros(self.vocab, dtype=bool), np.zeros(self.vocab)
            if "history" in names:
                seen[inside(self.history[b:e])] = True
                np.add.at(said, inside(self.history[a:e]), 1.0)
            rep = float(self.rep[r]) if "repetition" in names and self.rep[r] > 0 else 1.0
            f = float(self.freq[r]) if "frequency" in names and self.freq[r] == self.freq[r] else 0.0
            p = float(self.pres[r]) if "presence" in names and self.pres[r] == self.pres[r] else 0.0
            with np.errstate(invalid="ignore", over="ignore"):
                y[r] = np.where(seen, np.where(x[r] > 0, x[r] / rep, x[r] * rep), x[r])
                y[r] = np.where(said > 0, y[r] - f * said - p, y[r])
            size[r] = size[r] * max(rep, 1 / rep) + abs(f) * said + abs(p)
            if "bias_token" in names:
                t, v = self.bias_token[self.bias_at[r]:self.bias_at[r + 1]], self.bias_value[self.bias_at[r]:self.bias_at[r + 1]]
                keep = (t >= 0) & (t < self.vocab)
                np.add.at(y[r], t[keep], v[keep].astype(np.float64))
                np.add.at(size[r], t[keep], np.abs(v[keep]).astype(np.float64))
            if "allowed" in names and self.mask_row[r] >= 0:
                bits = np.unpackbits(self.masks[self.mask_row[r]].view(np.uint8), bitorder="little")[:self.vocab]
                y[r][bits == 0] = -np.inf
        return y, size

    def check(self, out, names, status=0):
        torch.cuda.synchronize()
        y, size = self.expected(names)
        got = out.double().cpu().numpy()
        assert np.array_equal(np.isneginf(got), np.isneginf(y)) and np.array_equal(np.isposinf(got), np.isposinf(y)) and np.array_equal(np.isnan(got), np.isnan(y))
        fin = np.isfinite(y)
        most = 6 + (np.diff(self.bias_at).max() if "bias_token" in names else 0)
        bound = np.where(fin, most * 2.0 ** -24 * size + (2.0 ** -8 * np.abs(np.where(fin, y, 0)) if self.dtype is BF16 else 0) + 1e-37, 0)
        assert (np.abs(np.where(fin, got - np.where(fin, y, 0), 0)) <= bound).all()
        # values that no rule names are the logits themselves
        assert int(self.status[0]) == status

    def run(self, drop=(), in_place=False, **change):
        a = self.args()
        for d in drop:
            for k in [k for k in a if k.startswith(d)]:
                a.pop(k)
        a.update(change)
        start = self.logits.clone()
        if in_place:
            work = torch.empty_strided(self.logits.shape, self.logits.stride(), dtype=self.dtype, device=gu.DEV).copy_(self.logits)
            kap.adjust_logits(work, device_status=self.status, **a)
            return work, a
        out = kap.adjust_logits(self.logits, self.out, device_status=self.status, **a)
        assert out is self.out and torch.equal(start.nan_to_num(1.0), self.logits.nan_to_num(1.0))
        return out, a


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype,pad,out_pad", [(F32, 0, 0), (F32, 3, 0), (F32, 1, 2), (BF16, 0, 0), (BF16, 15, 0), (BF16, 1, 8)])
@pytest.mark.parametrize("vocab", [1, 7, 31, 255, 1000, 50257])
def test_all_rules(vocab, dtype, pad, out_pad, in_place):
    c = Case(vocab, 6, vocab, dtype, pad, out_pad, masks=3)
    out, a = c.run(in_place=in_place)
    c.check(out, a)


@pytest.mark.parametrize("drop", [("history", "repetition", "presence", "frequency"), ("bias",), ("allowed",), ("history", "repetition", "presence", "frequency", "bias"),
                                  ("history", "repetition", "presence", "frequency", "allowed"), ("bias", "allowed"), ("repetition",), ("presence", "bias"),
                                  ("history", "repetition", "presence", "frequency", "bias", "allowed")])
@pytest.mark.parametrize("in_place", [False, True])
def test_each_rule_may_be_absent(drop, in_place):
    c = Case(3, 5, 3001, masks=2)
    out, a = c.run(drop, in_place)
    c.check(out, a)


def test_long_histories_and_many_rows():
    c = Case(4, 3, 128256, longest=100000, biases=3000, masks=2)
    out, a = c.run()
    c.check(out, a)
    c = Case(5, 300, 5000, BF16, longest=50, masks=7)
    out, a = c.run()
    c.check(out, a)


def test_largest_vocabulary():
    c = Case(6, 2, 811008, longest=3000, masks=1)
    out, a = c.run()
    c.check(out, a)
    with pytest.raises(kap.KapError) as e:
        kap.adjust_logits(torch.zeros(1, 811009, device=gu.DEV))
    assert e.value.code == kap.ERR_UNSUPPORTED


def test_infinities_and_nan():
    c = Case(7, 6, 900, masks=2)
    with torch.no_grad():
        for i, v in enumerate((float("inf"), -float("inf"), float("nan"), 3.4e38, -3.4e38, 0.0, -0.0, 1e-40)):
            c.logits[:, i::50] = v
    c.rep[:3] = 2.0
    out, a = c.run()
    y, _ = c.expected(a)
    with np.errstate(over="ignore"):
        far = np.abs(y) > 3.4028235e38
    got = out.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(y)) and np.array_equal(np.isneginf(got), np.isneginf(y) | (far & (y < 0)))
    out, a = c.run(in_place=True)
    assert np.array_equal(out.double().cpu().numpy(), got, equal_nan=True)


def test_parameters_that_switch_a_rule_off():
    c = Case(8, 6, 700)
    c.rep[:4] = [0.0, -1.0, np.nan, 1.0]
    c.pres[1:3] = np.nan
    c.freq[2:5] = np.nan
    out, a = c.run()
    c.check(out, a)


def test_rows_share_a_history():
    # a verification window: every row has one token more
    c = Case(9, 9, 500, longest=60)
    c.at[:] = [[3, 20, 20 + i] for i in range(9)]
    out, a = c.run()
    c.check(out, a)


def test_the_same_token_many_times():
    c = Case(10, 4, 5000, longest=3000)
    c.history[:] = 77
    c.bias_at = np.array([0, 3, 3, 5, 5], dtype=np.int32)
    c.bias_token, c.bias_value = np.array([77, 77, 77, 5, 77], dtype=np.int32), np.array([1e8, 1.0, -1e8, 2.0, 3.0], dtype=np.float32)
    first, a = c.run()
    c.check(first, a)
    first = first.clone()
    for _ in range(5):
        assert torch.equal(first, c.run()[0])


def test_tokens_outside_the_vocabulary_are_passed_over():
    c = Case(11, 3, 100, longest=50)
    c.history[::2] = 100
    c.history[1::4] = -5
    c.history[3::8] = 2 ** 31 - 1
    c.bias_at = np.array([0, 4, 4, 6], dtype=np.int32)
    c.bias_token, c.bias_value = np.array([-7, -7, 3, 100, 99, 2 ** 31 - 1], dtype=np.int32), np.arange(6, dtype=np.float32)
    out, a = c.run()
    c.check(out, a)


def test_what_is_reported():
    bit = 1 << kap.ERR_DEVICE_INDEX
    for bad in ([-1, 0, 5], [5, 4, 9], [0, 9, 4], [0, 1, 10 ** 9], [2 ** 62, 2 ** 62, 2 ** 62]):
        c = Case(12, 4, 300, masks=2)
        c.at[2] = bad
        out, a = c.run()
        c.at[2] = 0
        c.check(out, a, bit)
    for bad in (-2, 2, 2 ** 31 - 1):
        c = Case(13, 4, 300, masks=2)
        c.mask_row[1] = bad
        out, a = c.run()
        c.mask_row[1] = -1
        c.check(out, a, bit)
    for at in ([0, 2, 1, 3, 3], [0, 1, 2, 3, 99], [-1, 1, 2, 3, 3]):
        c = Case(14, 4, 300)
        c.bias_token, c.bias_value, c.bias_at = np.array([1, 2, 3], dtype=np.int32), np.ones(3, dtype=np.float32), np.array(at, dtype=np.int32)
        out, _ = c.run()
        torch.cuda.synchronize()
        assert int(c.status[0]) == bit
    c = Case(15, 1, 300)
    c.bias_token, c.bias_value, c.bias_at = np.array([9, 4], dtype=np.int32), np.ones(2, dtype=np.float32), np.array([0, 2], dtype=np.int32)
    c.run()
    torch.cuda.synchronize()
    assert int(c.status[0]) == bit


def test_in_place_writes_only_what_changes():
    c = Case(16, 4, 1000, pad=5, masks=2)
    store = torch.full((4, 1005), 9.0, device=gu.DEV)
    store[:, :1000] = c.logits
    a = c.args()
    kap.adjust_logits(store[:, :1000], device_status=c.status, **a)
    c.check(store[:, :1000], a)
    assert bool((store[:, 1000:] == 9.0).all())
    out = torch.full((4, 1009), 9.0, device=gu.DEV)
    kap.adjust_logits(c.logits, out[:, :1000], **a)
    c.check(out[:, :1000], a)
    assert bool((out[:, 1000:] == 9.0).all())


def test_captured_and_on_another_stream():
    c = Case(17, 5, 4000, masks=3)
    first, a = c.run()
    first = first.clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = torch.empty_like(first)
    kap.adjust_logits(c.logits, out, stream=side, **a)
    side.synchronize()
    assert torch.equal(first, out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kap.adjust_logits(c.logits, out, **a)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, out)


@pytest.mark.parametrize("in_place", [False, True])
def test_lists_without_entries(in_place):
    # the first step of a batch: nothing said yet, no biases; offsets that leave the empty lists are reported
    c = Case(53, 3, 500)
    empty = lambda t: torch.zeros(0, dtype=t, device=gu.DEV)                       # noqa: E731
    a = dict(c.args(), history=empty(torch.int32), history_at=torch.zeros(3, 3, dtype=torch.int64, device=gu.DEV), bias_indptr=torch.zeros(4, dtype=torch.int32, device=gu.DEV),
             bias_token=empty(torch.int32), bias_value=empty(F32), device_status=c.status)
    before = c.logits.clone()
    out = kap.adjust_logits(c.logits, None if in_place else c.out, **a)
    assert torch.equal(out, before) and int(c.status[0]) == 0
    a["history_at"][1, 2] = 1
    assert torch.equal(kap.adjust_logits(c.logits, None if in_place else c.out, **a), before)
    assert int(c.status[0]) == 1 << kap.ERR_DEVICE_INDEX
    c.status.zero_()
    a["history_at"].zero_()
    a["bias_indptr"][3] = 2
    assert torch.equal(kap.adjust_logits(c.logits, None if in_place else c.out, **a), before)
    assert int(c.status[0]) == 1 << kap.ERR_DEVICE_INDEX


def test_half_a_rule_is_refused():
    c = Case(54, 3, 100)
    a = c.args()
    for change in (dict(history=None), dict(history_at=None), dict(bias_indptr=None), dict(bias_token=None), dict(bias_value=None), dict(bias_token=None, bias_value=None)):
        with pytest.raises(kap.KapError) as e:
            kap.adjust_logits(c.logits, c.out, **{**a, **change})
        assert e.value.code == kap.ERR_INVALID_ARG
    assert bool((c.out == 7).all())


def test_calls_of_two_threads():
    # calls that need different amounts of shared memory, from two threads at once: both kernels of the shared-memory sizes that have to be asked for
    import threading
    cases = [Case(51, 128, 128256, longest=60, biases=0), Case(52, 128, 100000, longest=60, biases=0)]
    want = []
    for c in cases:
        c.arguments, c.stream = c.args(), torch.cuda.Stream()
        want.append(kap.adjust_logits(c.logits, c.out, **c.arguments).clone())
    torch.cuda.synchronize()
    failed = []

    def calls(c):
        try:
            torch.cuda.set_device(0)
            for _ in range(300):
                kap.adjust_logits(c.logits, c.out, **c.arguments, stream=c.stream)
            c.stream.synchronize()
        except Exception as e:                                                     # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=calls, args=(c,)) for c in cases]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for c, w in zip(cases, want):
        assert torch.equal(c.out, w)


def test_refusals():
    c = Case(18, 3, 100, masks=2)
    a = c.args()
    for change in (dict(history_at=None), dict(history=None), dict(bias_indptr=None), dict(bias_value=None), dict(allowed=None), dict(allowed_row=None),
                   dict(allowed=a["allowed"][:, :3]), dict(repetition=a["repetition"][:2]), dict(presence=a["presence"].double()), dict(history_at=a["history_at"].int()),
                   dict(bias_value=a["bias_value"][:-1]) if len(c.bias_token) else dict(bias_value=None)):
        with pytest.raises(kap.KapError) as e:
            kap.adjust_logits(c.logits, c.out, **{**a, **change})
        assert e.value.code == kap.ERR_INVALID_ARG
    for logits, out in ((c.logits.half(), None), (c.logits.cpu(), None), (c.logits.t(), None), (c.logits, c.out.bfloat16()), (c.logits, c.out[:2]), (c.logits[0], None)):
        with pytest.raises(kap.KapError):
            kap.adjust_logits(logits, out)
