"""Steps of a small two-layer model over a batch whose requests come and go: kap_build_block_tables gives the step its pages,
kap_append_kv_norm_rope places the new tokens, kap_chunk_attn reads them (one layer whole, one through a window), kap_adjust_logits and
kap_sample_tokens draw the next token of every sequence.  The attention of every step is held against a cache that is kept plainly, in 64 bits, the
rules and the draw against the single calls' definitions by their own tests; captured steps repeat the eager ones bit for bit."""
import numpy as np
import pytest
import torch

import gpu_util as gu
from paper_2607_24260_b200 import kap

pytestmark = pytest.mark.gpu
D, PAGE, HQ, HKV, VOCAB, WIDTH = 128, 16, 8, 2, 1003, 256
REQUESTS, ROWS, WINDOWS = 7, 160, [(0, 0), (40, 3)]
# (request, new tokens) of every step: prompts in chunks, single tokens, a request that ends and one that begins in its place
STEPS = [[(0, 100), (3, 7)], [(0, 60), (3, 1), (5, 33)], [(0, 1), (3, 1), (5, 1), (6, 90)], [(6, 1), (5, 1), (0, 1), (3, 1)], [(0, 1), (5, 1), (6, 1), (2, 17)],
         [(2, 1), (6, 1), (0, 1)]]
ENDS = {3: [3], 4: [5]}


class Server:
    def __init__(self):
        g = torch.Generator(device=gu.DEV).manual_seed(5)
        rand = lambda *s, by=1.0: torch.randn(s, device=gu.DEV, generator=g).mul_(by)     # noqa: E731
        bf = lambda t: t.to(torch.bfloat16)                                                # noqa: E731
        self.embed, self.head = bf(rand(VOCAB, WIDTH)), bf(rand(WIDTH, VOCAB, by=2 * WIDTH ** -0.5))
        self.qkv = [bf(rand(WIDTH, (HQ + 2 * HKV) * D, by=WIDTH ** -0.5)) for _ in WINDOWS]
        self.back = [bf(rand(HQ * D, WIDTH, by=(HQ * D) ** -0.5)) for _ in WINDOWS]
        self.qw, self.kw = bf(1 + rand(D, by=0.2)), bf(1 + rand(D, by=0.2))
        self.inv = (10000.0 ** (-torch.arange(D // 2, dtype=torch.float64) / (D // 2))).float().to(gu.DEV)
        self.pages = 80
        self.pool = [torch.full((self.pages, 2, HKV, PAGE, D), float("nan"), dtype=torch.bfloat16, device=gu.DEV) for _ in WINDOWS]
        self.state = dict(page_table=torch.full((REQUESTS, 20), -1, dtype=torch.int32, device=gu.DEV), pages_held=gu.i32([0] * REQUESTS),
                          free_pages=gu.i32(np.random.default_rng(1).permutation(self.pages)), free_count=gu.i32([self.pages]))
        self.ws = kap.Workspace(max_items=kap.chunk_attn_items(), max_rows_per_item=64, max_batch=REQUESTS)
        self.text = gu.i32(np.zeros(REQUESTS * 300))                                       # prompts and answers, 300 tokens a request
        self.status = torch.zeros(1, dtype=torch.int32, device=gu.DEV)
        batch = REQUESTS
        self.request, self.ctx, self.new = gu.i32(range(batch)), gu.i32([0] * batch), gu.i32([0] * batch)
        self.bt_indptr, self.bt_pages, self.new_indptr = gu.i32([0] * (batch + 1)), gu.i32([0] * 200), gu.i32([0] * (batch + 1))
        self.slot, self.position = torch.zeros(ROWS, dtype=torch.int64, device=gu.DEV), gu.i32([0] * ROWS)
        self.tokens, self.at = gu.i32([0] * ROWS), torch.zeros((batch, 3), dtype=torch.int64, device=gu.DEV)
        self.u = torch.zeros(batch, device=gu.DEV)
        f = lambda v: torch.full((batch,), v, device=gu.DEV)                               # noqa: E731
        self.rules = dict(repetition=f(1.2), presence=f(0.1), frequency=f(0.3), bias_indptr=gu.i32([2 * b for b in range(batch + 1)]),
                          bias_token=gu.i32([5, 900] * batch), bias_value=torch.tensor([1.5, -2.0] * batch, device=gu.DEV))
        bits = torch.randint(-2 ** 31, 2 ** 31 - 1, (2, (VOCAB + 31) // 32), generator=torch.Generator().manual_seed(2)).to(torch.int32)
        self.rules.update(allowed=bits.to(gu.DEV), allowed_row=gu.i32([0, -1, 1, -1, 0, -1, 1]))
        self.picked, self.logprob = gu.i32([0] * batch), torch.zeros(batch, device=gu.DEV)
        self.seen = []

    def step(self):
        """one step over the arrays as they are; all sizes are capacities, so it can be captured.  Unused sequences have no new tokens, and context 0."""
        kap.build_block_tables(self.ctx, **self.state, bt_indptr=self.bt_indptr, bt_pages=self.bt_pages, n_new=self.new, request=self.request,
                               new_indptr=self.new_indptr, slot=self.slot, position=self.position, device_status=self.status)
        x = self.embed[self.tokens.long()]
        total = self.ctx + self.new
        self.seen = []
        for i, (window, sink) in enumerate(WINDOWS):
            qkv = (x @ self.qkv[i]).view(ROWS, HQ + 2 * HKV, D)
            q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]
            q_rot = torch.zeros((ROWS, HQ, D), dtype=torch.bfloat16, device=gu.DEV)
            kap.append_kv_norm_rope(q, k, v, self.pool[i], self.bt_indptr, self.bt_pages, self.ctx, self.inv, self.qw, self.kw, q_out=q_rot,
                                    new_indptr=self.new_indptr, advance=False, device_status=self.status)
            out = torch.zeros_like(q_rot)
            kap.chunk_attn(q_rot, self.new_indptr, self.pool[i], self.bt_indptr, self.bt_pages, total, out, self.ws, window=window, n_sink=sink)
            self.seen.append((q, k, v, q_rot, out))
            x = (x + out.view(ROWS, -1) @ self.back[i])
        last = (self.new_indptr[1:].long() - 1).clamp(min=0)
        logits = (x[last] @ self.head).float()
        self.adjusted = kap.adjust_logits(logits, torch.empty_like(logits), history=self.text, history_at=self.at, device_status=self.status, **self.rules)
        kap.sample_tokens(self.adjusted, self.u, self.picked, self.logprob)
        self.ctx.copy_(total)

    def load(self, plan, lengths, texts, rng):
        pad = [r for r in range(REQUESTS) if r not in [p[0] for p in plan]]
        order = [p[0] for p in plan] + pad
        new = [p[1] for p in plan] + [0] * len(pad)
        self.request.copy_(gu.i32(order)), self.new.copy_(gu.i32(new))
        self.ctx.copy_(gu.i32([lengths[r] for r, _ in plan] + [0] * len(pad)))
        row, tokens = 0, np.zeros(ROWS, dtype=np.int64)
        for r, n in plan:
            tokens[row:row + n] = texts[r][lengths[r]:lengths[r] + n]
            row += n
        self.tokens.copy_(gu.i32(tokens))
        text, at = np.zeros((REQUESTS, 300), dtype=np.int64), np.zeros((REQUESTS, 3), dtype=np.int64)
        for b, r in enumerate(order):
            n = lengths[r] + new[b] if b < len(plan) else 0
            text[r, :n] = texts[r][:n]
            at[b] = [300 * r, 300 * r + n // 2, 300 * r + n]
        self.text.copy_(gu.i32(text.reshape(-1)))
        self.at.copy_(torch.from_numpy(at))
        self.u.copy_(torch.from_numpy(rng.random(REQUESTS).astype(np.float32)))


def _rotated(x, pos, inv):
    angle = pos.double()[:, None] * inv.double()
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = x[..., :D // 2], x[..., D // 2:]
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def _run(captured):
    s, rng = Server(), np.random.default_rng(11)
    lengths, texts = np.zeros(REQUESTS, dtype=np.int64), rng.integers(0, VOCAB, (REQUESTS, 300))
    cache = [[{} for _ in range(REQUESTS)] for _ in WINDOWS]                              # plain: the rows of k and v of every request
    graph, results = None, []
    if captured:
        # a step without rows, then the same captured
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            s.step()
        torch.cuda.current_stream().wait_stream(side)
        s.ctx.zero_()
        s.pool = [p.fill_(float("nan")) for p in s.pool]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.step()
        kept = s.seen
    for at, plan in enumerate(STEPS):
        s.load(plan, lengths, texts, rng)
        graph.replay() if captured else s.step()
        if captured:
            s.seen = kept
        torch.cuda.synchronize()
        s.ws.check()
        assert int(s.status[0]) == 0
        row = 0
        for b, (r, n) in enumerate(plan):
            pos = torch.arange(lengths[r], lengths[r] + n, device=gu.DEV)
            table = s.state["page_table"][r]
            assert torch.equal(s.slot[row:row + n], table[pos // PAGE].long() * PAGE + pos % PAGE)
            assert torch.equal(s.position[row:row + n].long(), pos)
            for i, (window, sink) in enumerate(WINDOWS):
                q, k, v, q_rot, out = (t[row:row + n] for t in s.seen[i])
                norm = lambda x, w: x.double() / (x.double().square().mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()       # noqa: E731
                for got, x, w in ((q_rot, q, s.qw), (s.pool[i][table[pos // PAGE].long(), 0, :, pos % PAGE], k, s.kw)):
                    y = _rotated(norm(x, w), pos, s.inv)
                    assert bool(((got.double() - y).abs() <= 2.0 ** -8 * y.abs() + 2.0 ** -16 * y.abs().amax(-1, keepdim=True)).all())
                kept_k = s.pool[i][table[pos // PAGE].long(), 0, :, pos % PAGE].double()
                was = cache[i][r]
                cache[i][r] = {"k": torch.cat([was["k"], kept_k]) if was else kept_k, "v": torch.cat([was["v"], v.double()]) if was else v.double()}
                keys, values = (cache[i][r][x].repeat_interleave(HQ // HKV, 1) for x in "kv")
                z = torch.einsum("nhd,thd->hnt", q_rot.double(), keys) * D ** -0.5
                t = torch.arange(len(keys), device=gu.DEV)
                sees = t[None] <= pos[:, None]
                if window:
                    sees &= (t[None] > pos[:, None] - window) | (t[None] < sink)
                w = torch.softmax(torch.where(sees, z, -torch.inf), -1)
                ref, size = torch.einsum("hnt,thd->nhd", w, values), torch.einsum("hnt,thd->nhd", w, values.abs())
                assert bool(((out.double() - ref).abs() <= 2.0 ** -8 * (size + ref.abs()) + 1e-3 * size).all())
            row += n
            lengths[r] += n
        for i in range(len(WINDOWS)):
            assert not bool(s.seen[i][4][row:].any())                                       # rows of nobody
        assert bool((s.picked[:len(plan)] >= 0).all())
        results.append([x.clone() for x in (s.adjusted[:len(plan)], s.picked[:len(plan)], s.logprob[:len(plan)], *s.state.values())])
        for b, (r, n) in enumerate(plan):                                                   # the drawn token is the text's next one
            texts[r, lengths[r]] = int(s.picked[b])
        if at in ENDS:
            kap.release_pages(gu.i32(ENDS[at]), **s.state)
            for r in ENDS[at]:
                lengths[r] = 0
                for i in range(len(WINDOWS)):
                    cache[i][r] = {}
    kap.release_pages(None, **s.state)
    assert int(s.state["free_count"][0]) == s.pages and sorted(s.state["free_pages"].tolist()) == list(range(s.pages))
    return results


def test_steps_eager_and_captured():
    eager, captured = _run(False), _run(True)
    for x, y in zip(eager, captured):
        for a, b in zip(x, y):
            assert torch.equal(a, b)
