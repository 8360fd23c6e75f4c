"""Four operators of a serving step that mixes chunks of prompts with single tokens, as cases to be timed and compared:
block tables built on the GPU, the append to the paged KV pool with normalised and rotated heads, attention of the new rows over the
paged cache (whole, or a sliding window with first tokens that stay visible), and penalties, biases and grammar masks on logits.

``own = False`` computes them in plain torch operations (32 bits, 64 for angles); ``own = True`` makes the calls of
``paper_2607_24260_b200.kap``.  Shapes: head dimension 128, pages of 16 tokens, the heads, context lengths and vocabulary of this
repository's workloads, and ranges around them.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
D, PAGE = 128, 16
VOCAB = 128256


# ------------------------------------------------------------------------------------------------- the cases
def listed():
    tables = dict(op="tables", ragged=3)
    append = dict(op="append", hq=32, hkv=8, rot=128, pairs="half", fused=True, layout="hnd", weights="shared")
    chunk = dict(op="chunk", hq=32, hkv=8, layout="hnd", window=0, sink=0, singles=0, ragged=0)
    logits = dict(op="logits", dtype="f32", pad=0, rules="penalties bias", grammar=0.0)
    return [
        # one token for each running request: latency
        dict(tables, name="tables 64 x 1 at 16K", batch=64, requests=256, new=1, ctx=16384),
        # a large server: many long contexts, some requests with a chunk of their prompt
        dict(tables, name="tables 512, chunks, to 128K", batch=512, requests=1024, new=512, ctx=131072),
        # one token of each running request, q, k and v as views of one fused projection
        dict(append, name="append 64 x 1 at 16K", batch=64, new=1, ctx=16384, ragged=0),
        # a chunk of prompts, separate projections, weights for each head, token-major pool, half of a head rotated
        dict(append, name="append 2 x 8192", batch=2, new=8192, ctx=4096, ragged=0, fused=False, weights="per head", layout="nhd", rot=64, pairs="even"),
        # the end of a prompt behind a cached document: latency
        dict(chunk, name="chunk 50 at 4K", batch=1, new=50, past=4096),
        # a step of a server: 60 requests with one token, four with a chunk of their prompt
        dict(chunk, name="chunk 4 x 512 + 60 x 1", batch=64, singles=60, new=512, past=16384, ragged=7),
        # a document being read: the last of its chunks
        dict(chunk, name="chunk 2048 at 128K", batch=1, new=2048, past=131072),
        # whole prompts of several lengths, nothing cached, token-major pool
        dict(chunk, name="prompts 3 x 5000, NHD", batch=3, new=5000, past=0, ragged=2, layout="nhd"),
        # windowed layers over contexts that have outgrown the window: single tokens and a few chunks
        dict(chunk, name="window 4096, 256 rows", batch=260, singles=256, new=1000, past=32768, window=4096, sink=16, ragged=5),
        # one row, a long history: latency
        dict(logits, name="logits 1 row", rows=1, vocab=VOCAB, history=20000, bias=100),
        # 16-bit logits, an odd vocabulary, rows with padding behind them, half of the rows under a grammar
        dict(logits, name="logits 64 bf16 rows, grammar", rows=64, vocab=50257, history=2000, bias=20, dtype="bf16", pad=15, grammar=0.5),
        # the verification windows of a large batch
        dict(logits, name="logits 512 rows", rows=512, vocab=VOCAB, history=4000, bias=10, grammar=0.1),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "append", "chunk", "chunk", "logits"])
    hkv = rng.choice([1, 2, 4, 8])
    heads = dict(hkv=hkv, hq=hkv * rng.choice([1, 2, 4, 8, 16] if hkv < 8 else [1, 2, 4, 8]), layout=rng.choice(["hnd", "nhd"]))
    ragged = rng.randrange(1, 1000)
    if op == "tables":
        batch = _log_uniform(rng, 1, 512)
        return dict(op=op, batch=batch, requests=batch + rng.randrange(0, 600), new=_log_uniform(rng, 1, 512), ctx=_log_uniform(rng, 1, 131072), ragged=ragged)
    if op == "append":
        batch = _log_uniform(rng, 1, 96)
        return dict(op=op, batch=batch, new=_log_uniform(rng, 1, max(1, 8192 // batch)), ctx=_log_uniform(rng, 1, 131072), ragged=ragged,
                    pairs=rng.choice(["half", "even"]), rot=rng.choice([32, 64, 96, 128]), fused=rng.random() < 0.5,
                    weights=rng.choice(["shared", "per head"]), **heads)
    if op == "chunk":
        singles = rng.choice([0, 0, _log_uniform(rng, 1, 128)])
        chunks = rng.randrange(0 if singles else 1, 5)
        batch = singles + chunks
        past = 0 if rng.random() < 0.2 and not singles else _log_uniform(rng, 64, 131072)
        past = min(past, max(16, (1 << 20) // batch))
        new = _log_uniform(rng, 2, 8192 // max(1, chunks))
        new = max(2, min(new, int(8e9 / (max(1, chunks) * (past + new) * max(1, heads["hq"] / 32)))))
        window = rng.choice([0, 0, _log_uniform(rng, 16, 16384)])
        return dict(op=op, batch=batch, singles=singles, new=new, past=past, window=window, sink=rng.choice([0, 4, 64]) if window else 0,
                    ragged=ragged, **heads)
    rows = _log_uniform(rng, 1, 400)
    return dict(op=op, rows=rows, vocab=_log_uniform(rng, 1000, 152064), history=_log_uniform(rng, 1, max(2, min(60000, 1500000 // rows))),
                bias=rng.choice([0, 5, 200]), dtype=rng.choice(["f32", "bf16"]), pad=rng.choice([0, 0, 3, 64]),
                rules=rng.choice(["penalties bias", "penalties", "bias"]), grammar=rng.choice([0.0, 0.3, 1.0]))


# ------------------------------------------------------------------------- sizes that a case stands for (host)
def _new_and_ctx(case):
    """new tokens and cached tokens of each sequence of a tables or append case"""
    rng = random.Random(case["ragged"])
    batch, new = case["batch"], case["new"]
    if not case["ragged"]:
        return [new] * batch, [case["ctx"]] * batch
    if case["op"] == "tables":                                                    # one in eight has a chunk, the others a token
        n_new = [rng.randint(1, new) if new > 1 and rng.random() < 0.125 else 1 for _ in range(batch)]
        return n_new, [_log_uniform(rng, max(1, case["ctx"] // 32), case["ctx"]) for _ in range(batch)]
    return [rng.randint(max(1, new // 4), new) for _ in range(batch)], [rng.randint(case["ctx"] // 2, case["ctx"]) for _ in range(batch)]


def _chunk_sizes(case):
    """(query rows, context length with them) of each sequence: the chunks lie among the single tokens"""
    rng = random.Random(case["ragged"])
    batch, new, past = case["batch"], case["new"], case["past"]
    n_q = [1] * case["singles"] + [new] * (batch - case["singles"])
    if case["ragged"]:
        n_q = [n if n == 1 else rng.randint(max(2, n // 2), n) for n in n_q]
        rng.shuffle(n_q)
        return n_q, [n + (rng.randint(past // 8, past) if past else 0) for n in n_q]
    return n_q, [n + past for n in n_q]


def _seen_pages(case, n, length):
    """logical pages that any of the sequence's rows sees, ascending"""
    end = (length + PAGE - 1) // PAGE
    if not case["window"]:
        return list(range(end))
    first = max(0, length - n - case["window"] + 1) // PAGE
    return [p for p in range(end) if p >= first or p * PAGE < case["sink"]]


def work(case):
    if case["op"] == "tables":
        n_new, ctx = _new_and_ctx(case)
        pages, rows = sum((c + n + PAGE - 1) // PAGE for n, c in zip(n_new, ctx)), sum(n_new)
        taken = sum((c + n + PAGE - 1) // PAGE - (c + PAGE - 1) // PAGE for n, c in zip(n_new, ctx))
        # the way there (every list, slots, positions, taken pages) and the pages' way back
        return dict(bytes=8 * pages + 12 * rows + 16 * taken + 28 * case["batch"], flops=pages + rows)
    if case["op"] == "append":
        rows = sum(_new_and_ctx(case)[0])
        return dict(bytes=2 * rows * (case["hq"] + 2 * case["hkv"]) * D * 2, flops=rows * (case["hq"] + case["hkv"]) * (3 * case["rot"] + 4 * D))
    if case["op"] == "chunk":
        n_q, ctx = _chunk_sizes(case)
        seen = tokens = 0
        for n, length in zip(n_q, ctx):
            p = np.arange(length - n, length, dtype=np.int64)
            w, s = case["window"], case["sink"]
            seen += int((p + 1).sum() if not w else (np.minimum(p + 1, w) + np.clip(p + 1 - w, 0, s)).sum())
            first = max(0, length - n - w + 1) if w else 0
            tokens += length - first + min(s, first)
        rows = sum(n_q)
        return dict(bytes=tokens * 2 * case["hkv"] * D * 2 + rows * case["hq"] * (2 * D * 2 + 4), flops=4 * D * case["hq"] * seen)
    size = 4 if case["dtype"] == "f32" else 2
    return dict(bytes=case["rows"] * (2 * case["vocab"] * size + 4 * case["history"] + 8 * case["bias"] + case["vocab"] // 8 * case["grammar"]),
                flops=case["rows"] * (case["vocab"] + 4 * case["history"]))


# ----------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _indptr(counts):
    return [0] + np.cumsum(counts, dtype=np.int64).tolist()


def _normal(shape, scale, g):
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    flat = out.view(-1)
    for at in range(0, flat.numel(), 1 << 26):
        part = flat[at:at + (1 << 26)]
        part.copy_(torch.randn(part.shape, device=DEV, generator=g) * scale)
    return out


def _pool(pages, hkv, layout, g):
    return _normal((pages, 2, hkv, PAGE, D) if layout == "hnd" else (pages, 2, PAGE, hkv, D), 0.5, g)


def _prepare_tables(case, s, g):
    n_new, ctx = _new_and_ctx(case)
    batch, requests, wide = case["batch"], case["requests"], (case["ctx"] + case["new"] + PAGE - 1) // PAGE
    held = [(c + PAGE - 1) // PAGE for c in ctx]
    total = sum((c + n + PAGE - 1) // PAGE for n, c in zip(n_new, ctx))
    taken = total - sum(held)
    pages = total + 1000
    perm = torch.randperm(pages, device=DEV, generator=g).to(torch.int32)
    rows = torch.randperm(requests, device=DEV, generator=g)[:batch]
    table = torch.full((requests, wide), -1, dtype=torch.int32, device=DEV)
    held_t = torch.tensor(held, device=DEV)
    inside = torch.arange(wide, device=DEV) < held_t[:, None]
    mine = torch.full((batch, wide), -1, dtype=torch.int32, device=DEV)
    mine[inside] = perm[:sum(held)]
    table[rows] = mine
    held_all = torch.zeros(requests, dtype=torch.int32, device=DEV)
    held_all[rows] = held_t.to(torch.int32)
    free = torch.full((pages,), -1, dtype=torch.int32, device=DEV)
    free[:pages - sum(held)] = perm[sum(held):]
    s.update(page_table=table, pages_held=held_all, free_pages=free, free_count=_i32([pages - sum(held)]), request=rows.to(torch.int32),
             ctx_len=_i32(ctx), n_new=_i32(n_new), bt_indptr=torch.zeros(batch + 1, dtype=torch.int32, device=DEV),
             bt_pages=torch.full((total + 100,), -1, dtype=torch.int32, device=DEV), new_indptr=torch.zeros(batch + 1, dtype=torch.int32, device=DEV),
             slot=torch.full((sum(n_new),), -1, dtype=torch.int64, device=DEV), position=torch.full((sum(n_new),), -1, dtype=torch.int32, device=DEV),
             most_taken=taken, most_pages=max((c + n + PAGE - 1) // PAGE for n, c in zip(n_new, ctx)), total=total)


def _prepare_append(case, s, g):
    n_new, ctx = _new_and_ctx(case)
    rows, hq, hkv = sum(n_new), case["hq"], case["hkv"]
    # the pages of the context behind the new tokens are one shared page: nothing reads them here
    own_pages = [(c + n - 1) // PAGE - c // PAGE + 1 for c, n in zip(ctx, n_new)]
    pages = 1 + sum(own_pages)
    fresh = torch.randperm(pages - 1, device=DEV, generator=g).to(torch.int32) + 1
    table, at = [], 0
    for c, n in zip(ctx, own_pages):
        table += [torch.zeros(c // PAGE, dtype=torch.int32, device=DEV), fresh[at:at + n]]
        at += n
    s.update(pool=_pool(pages, hkv, case["layout"], g), bt_pages=torch.cat(table),
             bt_indptr=_i32(_indptr([c // PAGE + n for c, n in zip(ctx, own_pages)])), ctx_len=_i32(ctx),
             new_indptr=None if max(n_new) == 1 else _i32(_indptr(n_new)))
    if case["fused"]:
        qkv = _normal((rows, hq + 2 * hkv, D), 1.0, g)
        s.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:])
    else:
        s.update(q=_normal((rows, hq, D), 1.0, g), k=_normal((rows, hkv, D), 1.0, g), v=_normal((rows, hkv, D), 1.0, g))
    s["q_out"] = torch.empty((rows, hq, D), dtype=torch.bfloat16, device=DEV)
    half = case["rot"] // 2
    s["inv_freq"] = (500000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).float().to(DEV)
    per_head = case["weights"] == "per head"
    weight = lambda heads: (1.0 + 0.3 * torch.randn((heads, D) if per_head else (D,), device=DEV, generator=g)).to(torch.bfloat16)  # noqa: E731
    s.update(q_weight=weight(hq), k_weight=weight(hkv), eps=1e-6)


def _prepare_chunk(case, s, g):
    n_q, ctx = _chunk_sizes(case)
    rows, hq, hkv = sum(n_q), case["hq"], case["hkv"]
    # pages that no row sees have been given back: their entries name page 0, which nothing reads for them
    seen = [_seen_pages(case, n, c) for n, c in zip(n_q, ctx)]
    pages = 1 + sum(len(x) for x in seen)
    perm = torch.randperm(pages - 1, device=DEV, generator=g).to(torch.int32) + 1
    lengths = [(c + PAGE - 1) // PAGE for c in ctx]
    starts = _indptr(lengths)
    held = torch.from_numpy(np.concatenate([np.array(x, dtype=np.int64) + at for x, at in zip(seen, starts)])).to(DEV)
    table = torch.zeros(starts[-1], dtype=torch.int32, device=DEV)
    table[held] = perm
    s.update(pool=_pool(pages, hkv, case["layout"], g), q=_normal((rows, hq, D), 1.0, g), bt_pages=table, bt_indptr=_i32(starts),
             ctx_len=_i32(ctx), q_indptr=_i32(_indptr(n_q)), n_q=n_q, ctx=ctx, out=torch.empty((rows, hq, D), dtype=torch.bfloat16, device=DEV),
             lse=torch.empty((rows, hq), dtype=torch.float32, device=DEV))
    if own:  # the workspace that a program keeps for all layers and steps
        from paper_2607_24260_b200 import kap
        s["ws"] = kap.Workspace(max_items=kap.chunk_attn_items(max_rows_per_item=64), max_rows_per_item=64, max_batch=case["batch"])
        s["ws"].set_kv_layout(kap.KV_HND if case["layout"] == "hnd" else kap.KV_NHD)


def _prepare_logits(case, s, g):
    rows, vocab, most = case["rows"], case["vocab"], case["history"]
    store = torch.randn((rows, vocab + case["pad"]), device=DEV, generator=g) * 3.0
    s["logits"] = store.to(torch.float32 if case["dtype"] == "f32" else torch.bfloat16)[:, :vocab]
    s["out"] = torch.empty((rows, vocab), dtype=s["logits"].dtype, device=DEV)
    rand = lambda *shape: torch.rand(shape, device=DEV, generator=g)               # noqa: E731
    s.update(history=None, history_at=None, repetition=None, presence=None, frequency=None, bias_indptr=None, bias_token=None, bias_value=None,
             allowed=None, allowed_row=None, longest=most)
    if "penalties" in case["rules"]:
        # words of a text: few frequent ones, many rare ones; a buffer of its own for each request, as long as the longest may get
        words = (vocab ** rand(rows, most + 8)).long().clamp(0, vocab - 1)
        shuffle = torch.randperm(vocab, device=DEV, generator=g)
        s["history"] = shuffle[words].to(torch.int32).view(-1)
        first = torch.arange(rows, device=DEV) * (most + 8)
        length = (most * (0.5 + 0.5 * rand(rows))).long().clamp(min=1) if rows > 1 else torch.full((1,), most, device=DEV)
        s["history_at"] = torch.stack([first, first + (length * 0.7 * rand(rows)).long(), first + length], 1).contiguous()
        # requests of several kinds: each rule off for some
        kind = torch.arange(rows, device=DEV) % 4
        s.update(repetition=torch.where(kind == 3, 1.0, 1.0 + 0.5 * rand(rows)), presence=torch.where(kind == 2, 0.0, rand(rows)),
                 frequency=torch.where(kind == 1, 0.0, 0.5 * rand(rows)))
    if "bias" in case["rules"] and case["bias"]:
        n = min(case["bias"], vocab)
        step = vocab // n
        token = torch.arange(n, device=DEV) * step + (rand(rows, n) * step).long()
        s.update(bias_indptr=_i32([n * r for r in range(rows + 1)]), bias_token=token.to(torch.int32).view(-1), bias_value=(rand(rows, n) * 20 - 10).view(-1))
    if case["grammar"]:
        words, grammars = (vocab + 31) // 32, 8
        # a grammar allows a run of tokens here and there, seldom half of the vocabulary
        bits = torch.randint(-2**31, 2**31, (grammars, words), device=DEV, generator=g)
        for _ in range(2):
            bits &= torch.randint(-2**31, 2**31, (grammars, words), device=DEV, generator=g)
        s["allowed"] = torch.where(rand(grammars, words) < 0.3, bits, 0).to(torch.int32)
        which = torch.randint(0, grammars, (rows,), device=DEV, generator=g)
        s["allowed_row"] = torch.where(rand(rows) < case["grammar"], which, -1).to(torch.int32)


def prepare(case, seed):
    g, s = _generator(seed), dict(case)
    {"tables": _prepare_tables, "append": _prepare_append, "chunk": _prepare_chunk, "logits": _prepare_logits}[case["op"]](case, s, g)
    return s


# ------------------------------------------------------------------------------------------------------- runs
def run(s):
    if own:
        return _run_own(s)
    return {"tables": _plain_tables, "append": _plain_append, "chunk": _plain_chunk, "logits": _plain_logits}[s["op"]](s)


def _run_own(s):
    from paper_2607_24260_b200 import kap
    if s["op"] == "tables":
        # a step's tables, and the step taken back (as after rejected proposals): the pages it took return to where they were
        kap.build_block_tables(s["ctx_len"], s["page_table"], s["pages_held"], s["free_pages"], s["free_count"], s["bt_indptr"], s["bt_pages"],
                               n_new=s["n_new"], request=s["request"], new_indptr=s["new_indptr"], slot=s["slot"], position=s["position"])
        kap.release_pages(s["request"], s["page_table"], s["pages_held"], s["free_pages"], s["free_count"], keep_tokens=s["ctx_len"])
        return _tables_out(s)
    if s["op"] == "append":
        # ctx_len advances once a step, with the last layer's call: this is one of the others
        kap.append_kv_norm_rope(s["q"], s["k"], s["v"], s["pool"], s["bt_indptr"], s["bt_pages"], s["ctx_len"], s["inv_freq"],
                                q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"], q_out=s["q_out"], new_indptr=s["new_indptr"],
                                interleaved=s["pairs"] == "even", advance=False, kv_layout=kap.KV_HND if s["layout"] == "hnd" else kap.KV_NHD)
        return s["q_out"], s["pool"]
    if s["op"] == "chunk":
        kap.chunk_attn(s["q"], s["q_indptr"], s["pool"], s["bt_indptr"], s["bt_pages"], s["ctx_len"], s["out"], s["ws"], lse=s["lse"],
                       window=s["window"], n_sink=s["sink"])
        return s["out"], s["lse"]
    kap.adjust_logits(s["logits"], s["out"], history=s["history"], history_at=s["history_at"], repetition=s["repetition"], presence=s["presence"],
                      frequency=s["frequency"], bias_indptr=s["bias_indptr"], bias_token=s["bias_token"], bias_value=s["bias_value"],
                      allowed=s["allowed"], allowed_row=s["allowed_row"])
    return s["out"]


def _tables_out(s):
    return (s["bt_indptr"], s["bt_pages"], s["new_indptr"], s["slot"], s["position"], s["page_table"], s["pages_held"], s["free_pages"], s["free_count"])


def _plain_tables(s):
    request, ctx, n_new = s["request"].long(), s["ctx_len"].long(), s["n_new"].long()
    table, held_all, free, count = s["page_table"], s["pages_held"], s["free_pages"], s["free_count"].long()
    held = held_all[request].long()
    pages = (ctx + n_new + PAGE - 1) // PAGE
    take = (pages - held).clamp(min=0)
    upto = take.cumsum(0)
    # taken pages, from the top of the stack downwards
    i = torch.arange(s["most_taken"], device=DEV)
    seq = torch.searchsorted(upto, i, right=True)
    logical = held[seq] + i - (upto - take)[seq]
    taken = free[count - 1 - i]
    table[request[seq], logical] = taken
    held_all[request] = torch.maximum(held, pages).to(torch.int32)
    s["free_count"].copy_(count - upto[-1])
    # the lists
    list_upto = pages.cumsum(0)
    i = torch.arange(s["total"], device=DEV)
    seq = torch.searchsorted(list_upto, i, right=True)
    s["bt_pages"][:s["total"]] = table[request[seq], i - (list_upto - pages)[seq]]
    s["bt_indptr"][1:] = list_upto
    new_upto = n_new.cumsum(0)
    s["new_indptr"][1:] = new_upto
    i = torch.arange(s["slot"].numel(), device=DEV)
    seq = torch.searchsorted(new_upto, i, right=True)
    pos = ctx[seq] + i - (new_upto - n_new)[seq]
    s["position"].copy_(pos)
    s["slot"].copy_(table[request[seq], pos // PAGE].long() * PAGE + pos % PAGE)
    # and back
    held, keep = held_all[request].long(), (ctx + PAGE - 1) // PAGE
    give = (held - keep).clamp(min=0)
    upto, count = give.cumsum(0), s["free_count"].long()
    i = torch.arange(s["most_taken"], device=DEV)
    seq = torch.searchsorted(upto, i, right=True)
    free[count + upto[-1] - 1 - i] = table[request[seq], keep[seq] + i - (upto - give)[seq]]
    held_all[request] = torch.minimum(held, keep).to(torch.int32)
    s["free_count"].copy_(count + upto[-1])
    return _tables_out(s)


def _rows_of(indptr, rows):
    """sequence and place in it of every row"""
    at = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(indptr.long(), at, right=True) - 1
    return seq, at - indptr.long()[seq]


def _norm(x, weight, eps):
    x = x.float()
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * weight.float()


def _rotate(x, cos, sin, rot, pairs):
    """x [rows, heads, D] in 32 bits; cos and sin [rows, rot / 2]"""
    c, s = cos[:, None, :], sin[:, None, :]
    turned, rest = x[..., :rot], x[..., rot:]
    if pairs == "half":
        a, b = turned[..., :rot // 2], turned[..., rot // 2:]
        return torch.cat([a * c - b * s, b * c + a * s, rest], -1)
    a, b = turned[..., 0::2], turned[..., 1::2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), rest], -1)


def _plain_append(s):
    rows, pool = s["q"].shape[0], s["pool"]
    if s["new_indptr"] is None:
        seq, place = torch.arange(rows, device=DEV), torch.zeros(rows, dtype=torch.int64, device=DEV)
    else:
        seq, place = _rows_of(s["new_indptr"], rows)
    at = s["ctx_len"].long()[seq] + place
    angle = at[:, None].double() * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _rotate(_norm(s["q"], s["q_weight"], s["eps"]), cos, sin, s["rot"], s["pairs"])
    k = _rotate(_norm(s["k"], s["k_weight"], s["eps"]), cos, sin, s["rot"], s["pairs"])
    page = s["bt_pages"].long()[s["bt_indptr"].long()[seq] + at // PAGE]
    s["q_out"].copy_(q)
    kv = torch.stack([k.bfloat16(), s["v"]], 1)                                   # [rows, 2, Hkv, D]
    if s["layout"] == "hnd":
        pool.permute(0, 3, 1, 2, 4)[page, at % PAGE] = kv
    else:
        pool.permute(0, 2, 1, 3, 4)[page, at % PAGE] = kv
    return s["q_out"], pool


def _plain_chunk(s):
    hkv, share, w, n_sink = s["hkv"], s["hq"] // s["hkv"], s["window"], s["sink"]
    pool = s["pool"] if s["layout"] == "hnd" else s["pool"].transpose(2, 3)       # [pages, 2, Hkv, 16, D]
    row = page_at = 0
    for n, length in zip(s["n_q"], s["ctx"]):
        first = max(0, length - n - w + 1) // PAGE if w else 0                    # pages before it matter for the sink only
        head = min(first, (n_sink + PAGE - 1) // PAGE)
        end = (length + PAGE - 1) // PAGE
        logical = torch.cat([torch.arange(head, device=DEV), torch.arange(first, end, device=DEV)])
        pages = s["bt_pages"][page_at + logical].long()
        t = (logical[:, None] * PAGE + torch.arange(PAGE, device=DEV)).view(-1)
        p = torch.arange(length - n, length, device=DEV)
        for lo in range(0, n, 1024):
            hi = min(n, lo + 1024)
            hidden = t > p[lo:hi, None]
            if w:
                hidden |= (t <= p[lo:hi, None] - w) & (t >= n_sink)
            some = hkv if (hi - lo) * s["hq"] * t.numel() < 1 << 31 else 1        # KV heads at a time
            for h in range(0, hkv, some):
                k, v = (pool[pages, part, h:h + some].transpose(0, 1).reshape(some, -1, D).float() for part in (0, 1))
                q = s["q"][row + lo:row + hi, h * share:(h + some) * share].float() * D ** -0.5
                q = q.view(hi - lo, some, share, D).permute(1, 2, 0, 3).reshape(some, -1, D)
                z = (q @ k.transpose(1, 2)).view(some, share, hi - lo, -1)
                z.masked_fill_(hidden, -math.inf)
                m = z.amax(-1, keepdim=True)
                z = z.sub_(m).exp_()
                total = z.sum(-1, keepdim=True)
                o = (z.view(some, share * (hi - lo), -1) @ v).view(some, share, hi - lo, D) / total
                s["out"][row + lo:row + hi, h * share:(h + some) * share] = o.permute(2, 0, 1, 3).reshape(hi - lo, -1, D).bfloat16()
                s["lse"][row + lo:row + hi, h * share:(h + some) * share] = (m + total.log())[..., 0].permute(2, 0, 1).reshape(hi - lo, -1)
        row += n
        page_at += end
    return s["out"], s["lse"]


def _plain_logits(s):
    x = s["logits"].float()
    rows, vocab = x.shape
    if s["history"] is not None:
        begin, answer, end = s["history_at"].unbind(1)
        at = begin[:, None] + torch.arange(s["longest"], device=DEV)
        token = s["history"][at.clamp(max=s["history"].numel() - 1)].long()
        count = torch.zeros((rows, vocab), device=DEV).scatter_add_(1, token, ((at >= answer[:, None]) & (at < end[:, None])).float())
        there = torch.zeros((rows, vocab), device=DEV).scatter_add_(1, token, (at < end[:, None]).float()) > 0
        r = s["repetition"][:, None]
        x = torch.where(there, torch.where(x > 0, x / r, x * r), x)
        x = x - s["frequency"][:, None] * count - s["presence"][:, None] * (count > 0)
    if s["bias_token"] is not None:
        x = x.scatter_add(1, s["bias_token"].view(rows, -1).long(), s["bias_value"].view(rows, -1))
    if s["allowed"] is not None:
        bits = s["allowed"][s["allowed_row"].clamp(min=0).long()]
        open_ = (bits[:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)).view(rows, -1)[:, :vocab] & 1
        x = torch.where((open_ == 1) | (s["allowed_row"] < 0)[:, None], x, -math.inf)
    s["out"].copy_(x)
    return s["out"]


# ------------------------------------------------------- what the definitions give in 64 bits, written on their own
def exact(case, seed):
    if case["op"] == "tables":                                                    # whole numbers
        return None
    s = _inputs_only(case, seed)
    return {"append": _exact_append, "chunk": _exact_chunk, "logits": _exact_logits}[case["op"]](case, s)


def _inputs_only(case, seed):
    """prepare() without the handle of the framework, whatever ``own`` says"""
    global own
    before, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = before


def _exact_append(case, s):
    n_new, ctx = _new_and_ctx(case)
    half = case["rot"] // 2
    first = [(i, i + half) if case["pairs"] == "half" else (2 * i, 2 * i + 1) for i in range(half)]
    a, b = (torch.tensor([p[j] for p in first], device=DEV) for j in (0, 1))
    pos = torch.cat([torch.arange(c, c + n, device=DEV) for c, n in zip(ctx, n_new)])
    # exp(i angle) as complex numbers
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos[:, None].double() * s["inv_freq"].double())[:, None, :]

    def turned(x, weight):
        x = x.double()
        x = x / torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / D + case_eps) * weight.double()
        y = torch.complex(x[..., a], x[..., b]) * turn
        x[..., a], x[..., b] = y.real, y.imag
        return x

    case_eps = s["eps"]
    pool = s["pool"].double()
    k, v = turned(s["k"], s["k_weight"]), s["v"].double()
    row = 0
    for i, (c, n) in enumerate(zip(ctx, n_new)):
        t = torch.arange(c, c + n, device=DEV)
        page = s["bt_pages"][int(s["bt_indptr"][i]) + t // PAGE].long()
        for part, x in ((0, k), (1, v)):
            for h in range(case["hkv"]):
                to = (page, part, h, t % PAGE) if case["layout"] == "hnd" else (page, part, t % PAGE, h)
                pool[to] = x[row:row + n, h]
        row += n
    return turned(s["q"], s["q_weight"]), pool


def _exact_chunk(case, s):
    if work(case)["flops"] > 6e12:
        return None
    n_q, ctx = _chunk_sizes(case)
    rows, share = sum(n_q), case["hq"] // case["hkv"]
    out = torch.empty((rows, case["hq"], D), dtype=torch.float64, device=DEV)
    lse = torch.empty((rows, case["hq"]), dtype=torch.float64, device=DEV)
    heads_first = s["pool"] if case["layout"] == "hnd" else s["pool"].transpose(2, 3)
    starts, r0 = s["bt_indptr"].tolist(), 0
    for b, (n, length) in enumerate(zip(n_q, ctx)):
        table = s["bt_pages"][starts[b]:starts[b + 1]].long()
        for lo in range(0, n, 256):
            hi = min(n, lo + 256)
            p = torch.arange(length - n + lo, length - n + hi, device=DEV)
            # the tokens that one of these rows sees, and who sees them
            t = torch.arange(length - n + hi, device=DEV)
            if case["window"]:
                t = t[(t < case["sink"]) | (t > length - n + lo - case["window"])]
            behind = p[:, None] - t[None, :]
            sees = behind >= 0
            if case["window"]:
                sees &= (behind < case["window"]) | (t < case["sink"])[None, :]
            for h in range(case["hkv"]):
                k, v = (heads_first[table[t // PAGE], part, h, t % PAGE].double() for part in (0, 1))
                q = s["q"][r0 + lo:r0 + hi, h * share:(h + 1) * share].double() / math.sqrt(D)
                z = torch.einsum("rgd,td->rgt", q, k)
                z = torch.where(sees[:, None], z, -math.inf)
                total = torch.logsumexp(z, -1)
                lse[r0 + lo:r0 + hi, h * share:(h + 1) * share] = total
                out[r0 + lo:r0 + hi, h * share:(h + 1) * share] = torch.einsum("rgt,td->rgd", (z - total[..., None]).exp(), v)
        r0 += n
    return out, lse


def _exact_logits(case, s):
    """Row by row, from the rules."""
    rows, vocab = case["rows"], case["vocab"]
    out = s["logits"].double()
    for r in range(rows):
        if s["history"] is not None:
            begin, answer, end = s["history_at"][r].tolist()
            said = torch.bincount(s["history"][answer:end], minlength=vocab).double()
            known = torch.zeros(vocab, dtype=torch.bool, device=DEV)
            known[s["history"][begin:end].long()] = True
            factor = float(s["repetition"][r])
            x = out[r].clone()
            x[known & (out[r] > 0)] /= factor
            x[known & (out[r] <= 0)] *= factor
            out[r] = x - float(s["frequency"][r]) * said - float(s["presence"][r]) * (said > 0)
        if s["bias_token"] is not None:
            i, j = s["bias_indptr"][r:r + 2].tolist()
            out[r, s["bias_token"][i:j].long()] += s["bias_value"][i:j].double()
        if s["allowed"] is not None and int(s["allowed_row"][r]) >= 0:
            words = s["allowed"][int(s["allowed_row"][r])].cpu().numpy().view(np.uint8)
            closed = np.unpackbits(words, bitorder="little")[:vocab] == 0
            out[r, torch.from_numpy(closed).to(DEV)] = -math.inf
    return out
