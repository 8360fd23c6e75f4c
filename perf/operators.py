"""Three operators of a decoding step, as cases to be timed and compared: appending rotated keys to the paged KV
pool, attention over a batch that shares a long prefix, and sampling the next token.

``own = False`` computes them in plain torch operations (32 bits, 64 where a value may sit next to a border);
``own = True`` makes the calls of ``paper_2607_24260_b200.kap``.  Shapes: head dimension 128, pages of 16 tokens, the
heads, context lengths and vocabulary of this repository's workloads, and ranges around them.
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
    append = dict(op="append", hq=32, hkv=8, rot=128, axes=1, pairs="half", fused=True, layout="hnd")
    prefix = dict(op="prefix", hq=32, hkv=8, layout="hnd", groups=1, ragged=0)
    sample = dict(op="sample", dtype="f32", pad=0, spread=2.5)
    return [
        # one proposal step of a small batch: latency
        dict(append, name="append 4 x 1 at 128K", batch=4, new=1, ctx=131072, ragged=0),
        # one step of a full batch, q, k and v as views of one fused projection
        dict(append, name="append 64 x 1 at 16K", batch=64, new=1, ctx=16384, ragged=0),
        # image and text positions on three axes, interleaved pairs, half of the head rotated, token-major pool, ragged windows
        dict(append, name="append 3-axis ragged", batch=24, new=200, ctx=9000, ragged=5, axes=3, pairs="even", rot=64, layout="nhd"),
        # a chunk of prompts being filled in
        dict(append, name="append 2 x 8192", batch=2, new=8192, ctx=4096, ragged=0, fused=False),
        # a short instruction shared by a few requests: latency
        dict(prefix, name="prefix 512, 4 sequences", batch=4, prefix=512, suffix=64, n_q=1),
        # a shared document, every request with a dialogue of its own
        dict(prefix, name="prefix 32K, 64 sequences", batch=64, prefix=32768, suffix=512, n_q=1),
        # four documents, groups and windows of several sizes, token-major pool
        dict(prefix, name="4 prefixes, ragged windows", batch=48, prefix=16384, suffix=900, n_q=8, groups=4, ragged=3, layout="nhd"),
        # verification windows of a whole batch over the longest context
        dict(prefix, name="prefix 128K, 64 x 4 rows", batch=64, prefix=131072, suffix=1024, n_q=4),
        # one row: latency
        dict(sample, name="sample 1 row", rows=1, vocab=VOCAB, filters="top_k top_p"),
        # a batch in which every request has its own settings, some greedy
        dict(sample, name="sample 64 rows, mixed", rows=64, vocab=VOCAB, filters="mixed"),
        # 16-bit logits, an odd vocabulary, rows with padding behind them, a nearly flat distribution
        dict(sample, name="sample 100 bf16 rows, top_p", rows=100, vocab=50257, filters="top_p", dtype="bf16", pad=15, spread=1.0),
        # the verification windows of a large batch, plain temperature
        dict(sample, name="sample 512 rows", rows=512, vocab=VOCAB, filters="none"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "prefix", "sample"])
    hkv = rng.choice([2, 4, 8])
    heads = dict(hkv=hkv, hq=hkv * rng.choice([1, 2, 4, 8]) if op == "append" else hkv * rng.choice([4, 8]))
    if op == "append":
        batch = _log_uniform(rng, 1, 96)
        return dict(op=op, batch=batch, new=_log_uniform(rng, 1, max(1, 8192 // batch)), ctx=_log_uniform(rng, 1, 131072),
                    ragged=rng.randrange(1, 1000), axes=rng.choice([1, 3]), pairs=rng.choice(["half", "even"]),
                    rot=rng.choice([32, 64, 96, 128]), fused=rng.random() < 0.5, layout=rng.choice(["hnd", "nhd"]), **heads)
    if op == "prefix":
        batch = rng.randrange(2, 65)
        n_q = _log_uniform(rng, 1, 8)
        most = max(64, min(131072, 131072 * 256 * 32 // (batch * n_q * heads["hq"]) // 2))
        return dict(op=op, batch=batch, prefix=PAGE * max(1, _log_uniform(rng, 64, most) // PAGE), suffix=_log_uniform(rng, 16, 1024), n_q=n_q,
                    groups=rng.choice([1, 1, 2, 5]), ragged=rng.randrange(1, 1000), layout=rng.choice(["hnd", "nhd"]), **heads)
    rows = _log_uniform(rng, 1, 400)
    return dict(op=op, rows=rows, vocab=_log_uniform(rng, 1000, 152064), filters=rng.choice(["none", "top_k", "top_p", "min_p", "top_k top_p", "mixed"]),
                dtype=rng.choice(["f32", "bf16"]), pad=rng.choice([0, 0, 3, 64]), spread=rng.choice([0.7, 1.5, 2.5, 4.0]))


# ------------------------------------------------------------------------- sizes that a case stands for (host)
def _append_sizes(case):
    rng = random.Random(case["ragged"])
    batch, new = case["batch"], case["new"]
    if not case["ragged"]:
        return [new] * batch, [case["ctx"]] * batch
    return [rng.randint(max(1, new // 4), new) for _ in range(batch)], [rng.randint(case["ctx"] // 2, case["ctx"]) for _ in range(batch)]


def _prefix_sizes(case):
    """(first sequence of each group and the end, prefix tokens of each group, rows and own tokens of each sequence)"""
    rng = random.Random(case["ragged"])
    batch, groups = case["batch"], min(case["groups"], case["batch"])
    cuts = [0] + sorted(rng.sample(range(1, batch), groups - 1)) + [batch]
    prefix, n_q, tail = [case["prefix"]] * groups, [case["n_q"]] * batch, [case["suffix"]] * batch
    if case["ragged"]:
        prefix = [PAGE * rng.randint((case["prefix"] // PAGE + 1) // 2, case["prefix"] // PAGE) for _ in range(groups)]
        n_q = [rng.randint(max(1, case["n_q"] // 2), case["n_q"]) for _ in range(batch)]
    tail = [max(n, _log_uniform(rng, max(1, t // 16), t)) for n, t in zip(n_q, tail)]
    return cuts, prefix, n_q, tail


def work(case):
    if case["op"] == "append":
        n_new, _ = _append_sizes(case)
        rows = sum(n_new)
        moved = 2 * rows * (case["hq"] + 2 * case["hkv"]) * D * 2
        return dict(bytes=moved, flops=3 * rows * (case["hq"] + case["hkv"]) * case["rot"])
    if case["op"] == "prefix":
        cuts, prefix, n_q, tail = _prefix_sizes(case)
        rows, token = sum(n_q), 2 * case["hkv"] * D * 2
        seen = sum(sum(n_q[b] * (p + tail[b]) for b in range(cuts[g], cuts[g + 1])) for g, p in enumerate(prefix))
        return dict(bytes=(sum(prefix) + sum(tail)) * token + rows * case["hq"] * (2 * D * 2 + 4), flops=4 * D * case["hq"] * seen)
    size = 4 if case["dtype"] == "f32" else 2
    return dict(bytes=case["rows"] * (case["vocab"] * size + 24), flops=4 * case["rows"] * case["vocab"])


# ----------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _indptr(counts):
    return [0] + list(np.cumsum(counts, dtype=np.int64).tolist())


def _normal(shape, scale, g):
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    flat = out.view(-1)
    for at in range(0, flat.numel(), 1 << 26):
        part = flat[at:at + (1 << 26)]
        part.copy_(torch.randn(part.shape, device=DEV, generator=g) * scale)
    return out


def _pool(pages, hkv, layout, g):
    return _normal((pages, 2, hkv, PAGE, D) if layout == "hnd" else (pages, 2, PAGE, hkv, D), 0.5, g)


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case)
    if case["op"] == "append":
        n_new, ctx = _append_sizes(case)
        rows, hq, hkv = sum(n_new), case["hq"], case["hkv"]
        # the pages of the context behind the window are one shared page: nothing reads them here
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
        s["positions"], s["freq_axis"] = None, None
        if case["axes"] > 1:
            # time advances slowly, height and width walk over images of 24 x 36 patches
            i = torch.arange(rows, device=DEV)
            base = torch.randint(0, 4000, (1,), device=DEV, generator=g)
            s["positions"] = torch.stack([base + i // 864, base + i // 36 % 24, base + i % 36]).to(torch.int32)
            s["freq_axis"] = [0 if f < half // 4 else 1 + (f - half // 4) % 2 for f in range(half)]
    elif case["op"] == "prefix":
        cuts, prefix, n_q, tail = _prefix_sizes(case)
        batch, rows, hq, hkv = case["batch"], sum(n_q), case["hq"], case["hkv"]
        own_pages = [(t + PAGE - 1) // PAGE for t in tail]
        pages = sum(prefix) // PAGE + sum(own_pages)
        perm = torch.randperm(pages, device=DEV, generator=g).to(torch.int32)
        shared = perm[:sum(prefix) // PAGE].split([p // PAGE for p in prefix])
        mine = perm[sum(prefix) // PAGE:].split(own_pages)
        group = [i for i in range(len(prefix)) for _ in range(cuts[i], cuts[i + 1])]
        s.update(pool=_pool(pages, hkv, case["layout"], g), q=_normal((rows, hq, D), 1.0, g),
                 bt_pages=torch.cat([x for b in range(batch) for x in (shared[group[b]], mine[b])]),
                 bt_indptr=_i32(_indptr([prefix[group[b]] // PAGE + own_pages[b] for b in range(batch)])),
                 ctx_len=_i32([prefix[group[b]] + tail[b] for b in range(batch)]), q_indptr=_i32(_indptr(n_q)),
                 n_q=np.array(n_q, dtype=np.int32), group_indptr=np.array(cuts, dtype=np.int32),
                 prefix_pages=np.array([p // PAGE for p in prefix], dtype=np.int32), longest_tail=max(tail),
                 list_len=np.array([prefix[group[b]] // PAGE + own_pages[b] for b in range(batch)], dtype=np.int32),
                 out=torch.empty((rows, hq, D), dtype=torch.bfloat16, device=DEV), lse=torch.empty((rows, hq), dtype=torch.float32, device=DEV))
        if own:  # the schedule that a program keeps for all layers of a step
            from paper_2607_24260_b200 import kap
            s["ws"] = kap.Workspace(max_items=kap.shared_prefix_items(s["list_len"], s["n_q"], s["group_indptr"], s["prefix_pages"], hq, hkv),
                                    max_rows_per_item=64, max_batch=batch)
            s["ws"].set_kv_layout(kap.KV_HND if case["layout"] == "hnd" else kap.KV_NHD)
            s["ws"].schedule_shared_prefix(s["list_len"], s["n_q"], s["group_indptr"], s["prefix_pages"], hq, hkv)
    else:
        rows, vocab = case["rows"], case["vocab"]
        store = torch.randn((rows, vocab + case["pad"]), device=DEV, generator=g) * case["spread"]
        # a head of likely tokens over a broad bulk
        likely = torch.randint(0, vocab, (rows, 40), device=DEV, generator=g)
        lift = 11.0 - 2.0 * torch.log1p(torch.arange(40, device=DEV, dtype=torch.float32))
        store.scatter_add_(1, likely, lift.expand(rows, 40) * min(1.0, case["spread"] / 2))
        store = store.to(torch.float32 if case["dtype"] == "f32" else torch.bfloat16)
        f, n = case["filters"], torch.rand((5, rows), device=DEV, generator=g)
        s.update(logits=store[:, :vocab], uniform=n[0].contiguous(), temperature=(0.6 + 0.7 * n[1]).contiguous(), top_k=None, top_p=None, min_p=None)
        if "top_k" in f or f == "mixed":
            s["top_k"] = (1 + (n[2] * 80)).to(torch.int32)
        if "top_p" in f or f == "mixed":
            s["top_p"] = (0.8 + 0.19 * n[3]).contiguous()
        if "min_p" in f or f == "mixed":
            s["min_p"] = (0.02 + 0.1 * n[4]).contiguous()
        if f == "mixed":  # requests of several kinds in one batch: each filter off for some rows, some rows greedy
            kind = torch.arange(rows, device=DEV)
            s["temperature"] = torch.where(kind % 8 == 3, 0.0, s["temperature"])
            s["top_k"] = torch.where(kind % 3 == 0, 0, s["top_k"]).to(torch.int32)
            s["top_p"] = torch.where(kind % 4 == 1, 1.0, s["top_p"])
            s["min_p"] = torch.where(kind % 2 == 0, 0.0, s["min_p"])
        s.update(token=torch.empty(rows, dtype=torch.int32, device=DEV), logprob=torch.empty(rows, dtype=torch.float32, device=DEV))
    return s


# ------------------------------------------------------------------------------------------------------- runs
def run(s):
    if own:
        return _run_own(s)
    return {"append": _plain_append, "prefix": _plain_prefix, "sample": _plain_sample}[s["op"]](s)


def _run_own(s):
    from paper_2607_24260_b200 import kap
    if s["op"] == "append":
        # ctx_len advances once a step, with the last layer's call: this is one of the others
        kap.append_kv_rope(s["q"], s["k"], s["v"], s["pool"], s["bt_indptr"], s["bt_pages"], s["ctx_len"], s["inv_freq"], s["q_out"],
                           new_indptr=s["new_indptr"], positions=s["positions"], freq_axis=s["freq_axis"], interleaved=s["pairs"] == "even",
                           advance=False, kv_layout=kap.KV_HND if s["layout"] == "hnd" else kap.KV_NHD)
        return s["q_out"], s["pool"]
    if s["op"] == "prefix":
        kap.shared_prefix_attn(s["q"], s["q_indptr"], s["pool"], s["bt_indptr"], s["bt_pages"], s["ctx_len"], s["out"], s["ws"], lse=s["lse"])
        return s["out"], s["lse"]
    kap.sample_tokens(s["logits"], s["uniform"], s["token"], s["logprob"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                      min_p=s["min_p"])
    return s["token"], s["logprob"]


def _rows_of(indptr, rows):
    """sequence and place in it of every row"""
    at = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(indptr.long(), at, right=True) - 1
    return seq, at - indptr.long()[seq]


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
    if s["positions"] is None:
        pos = at[:, None].expand(rows, s["rot"] // 2)
    else:
        pos = s["positions"].long().t()[:, torch.tensor(s["freq_axis"], device=DEV)]
    angle = pos.double() * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _rotate(s["q"].float(), cos, sin, s["rot"], s["pairs"])
    k = _rotate(s["k"].float(), cos, sin, s["rot"], s["pairs"])
    page = s["bt_pages"].long()[s["bt_indptr"].long()[seq] + at // PAGE]
    s["q_out"].copy_(q)
    kv = torch.stack([k.bfloat16(), s["v"]], 1)                                   # [rows, 2, Hkv, D]
    if s["layout"] == "hnd":
        pool.permute(0, 3, 1, 2, 4)[page, at % PAGE] = kv
    else:
        pool.permute(0, 2, 1, 3, 4)[page, at % PAGE] = kv
    return s["q_out"], pool


def _gather(pool, pages, layout, part):
    """K (part 0) or V (part 1) of the pages [n, m], in 32 bits: [n, Hkv, 16 m, D]"""
    x = pool[:, part] if layout == "hnd" else pool[:, part].transpose(1, 2)
    x = x[pages]                                                                  # [n, m, Hkv, 16, D]
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3).float()


def _plain_prefix(s):
    q, pool, hkv, rows = s["q"], s["pool"], s["hkv"], s["q"].shape[0]
    share = s["hq"] // hkv
    cuts = torch.from_numpy(s["group_indptr"]).to(DEV).long()
    pages = torch.from_numpy(s["prefix_pages"]).to(DEV).long()
    seq, place = _rows_of(s["q_indptr"], rows)
    group = torch.searchsorted(cuts, seq, right=True) - 1
    limit = s["ctx_len"].long()[seq] - (s["q_indptr"].long()[seq + 1] - s["q_indptr"].long()[seq]) + place  # last visible token
    table, starts = s["bt_pages"].long(), s["bt_indptr"].long()
    # the prefix, once a group: rows of the group padded to the largest group's
    n_groups, most = pages.numel(), int(s["prefix_pages"].max())
    first = s["q_indptr"].long()[cuts]                                            # first row of each group, and the end
    wide = int(max(np.add.reduceat(s["n_q"], s["group_indptr"][:-1])))
    g_rows = (first[:-1, None] + torch.arange(wide, device=DEV)).clamp(max=rows - 1)
    g_pages = table[(starts[cuts[:-1], None] + torch.arange(most, device=DEV)).clamp(max=table.numel() - 1)]
    q32 = q.float().view(rows, hkv, share, D) * D ** -0.5
    qg = q32[g_rows].permute(0, 2, 1, 3, 4).reshape(n_groups, hkv, wide * share, D)
    z1 = qg @ _gather(pool, g_pages, s["layout"], 0).transpose(-1, -2)            # [groups, Hkv, wide * share, 16 most]
    token = torch.arange(most * PAGE, device=DEV)
    z1.masked_fill_((token >= pages[:, None] * PAGE)[:, None, None, :], -math.inf)
    # every sequence's own tokens, padded to the longest
    longest = (s["longest_tail"] + PAGE - 1) // PAGE
    batch, nq = s["batch"], int(s["n_q"].max())
    s_rows = (s["q_indptr"].long()[:-1, None] + torch.arange(nq, device=DEV)).clamp(max=rows - 1)
    s_group = torch.searchsorted(cuts, torch.arange(batch, device=DEV), right=True) - 1
    s_pages = table[((starts[:-1] + pages[s_group])[:, None] + torch.arange(longest, device=DEV)).clamp(max=table.numel() - 1)]
    qs = q32[s_rows].permute(0, 2, 1, 3, 4).reshape(batch, hkv, nq * share, D)
    z2 = qs @ _gather(pool, s_pages, s["layout"], 0).transpose(-1, -2)
    pos = pages[s_group][:, None] * PAGE + torch.arange(longest * PAGE, device=DEV)
    hidden = pos[:, None, :] > limit[s_rows][:, :, None]                          # [batch, nq, tokens]
    z2.masked_fill_(hidden.repeat_interleave(share, 1)[:, None], -math.inf)
    # one softmax over both parts
    at1 = (group, torch.arange(rows, device=DEV) - first[group])        # place of every row among the padded ones
    pick1 = lambda x: x.unflatten(2, (wide, share))[at1[0], :, at1[1]]            # noqa: E731  [rows, Hkv, share, ...]
    pick2 = lambda x: x.unflatten(2, (nq, share))[seq, :, place]                  # noqa: E731
    m = torch.maximum(pick1(z1.amax(-1)), pick2(z2.amax(-1)))                     # [rows, Hkv, share]
    m1 = m[g_rows].permute(0, 2, 1, 3).reshape(n_groups, hkv, -1, 1)
    m2 = m[s_rows].permute(0, 2, 1, 3).reshape(batch, hkv, -1, 1)
    z1, z2 = z1.sub_(m1).exp_(), z2.sub_(m2).exp_()
    total = pick1(z1.sum(-1)) + pick2(z2.sum(-1))
    v2 = _gather(pool, s_pages, s["layout"], 1)
    out = pick1(z1 @ _gather(pool, g_pages, s["layout"], 1)) + pick2(z2 @ v2)
    s["out"].copy_((out / total[..., None]).view(rows, -1, D))
    s["lse"].copy_((m + total.log()).view(rows, -1))
    return s["out"], s["lse"]


def _plain_sample(s):
    # 64 bits throughout: the token is decided by comparisons of long sums
    x = s["logits"].double()
    x = torch.where(x.isnan(), -math.inf, x)
    rows, vocab = x.shape
    top, place = x.amax(1, keepdim=True), torch.arange(vocab, device=DEV)
    best = torch.where(x == top, place, vocab).amin(1, keepdim=True)              # the lowest index among equals
    t = s["temperature"].double()[:, None]
    z = torch.where(x == top, 0.0, (x - top) / torch.where(t > 0, t, 1.0))
    w = z.exp()
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    ranked = w.gather(1, order)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        ranked = torch.where((place < k) | (k <= 0), ranked, 0.0)
    keep = ranked > 0
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        upto = ranked.cumsum(1)
        before = torch.cat([torch.zeros_like(upto[:, :1]), upto[:, :-1]], 1)
        keep &= (before < p * upto[:, -1:]) | (p >= 1) | (place == 0)
    if s["min_p"] is not None:
        keep &= z.gather(1, order) >= s["min_p"].double()[:, None].log()
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ranked, 0.0))
    upto = kept.cumsum(1)
    token = torch.searchsorted(upto, s["uniform"].double()[:, None] * upto[:, -1:], right=True).clamp(max=vocab - 1)
    greedy = ~(t > 0)
    token = torch.where(greedy, best, token)
    logprob = torch.where(greedy, 0.0, z.gather(1, token) - upto[:, -1:].log())
    dead = top == -math.inf
    s["token"].copy_(torch.where(dead, -1, token)[:, 0])
    s["logprob"].copy_(torch.where(dead, -math.inf, logprob)[:, 0])
    return s["token"], s["logprob"]


# ------------------------------------------------------- what the definitions give in 64 bits, written on their own
def exact(case, seed):
    s = prepare_inputs_only(case, seed)
    return {"append": _exact_append, "prefix": _exact_prefix, "sample": _exact_sample}[case["op"]](case, s)


def prepare_inputs_only(case, seed):
    """prepare() without the handle of the framework, whatever ``own`` says"""
    global own
    before, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = before


def _exact_append(case, s):
    n_new, ctx = _append_sizes(case)
    half = case["rot"] // 2
    first = [(i, i + half) if case["pairs"] == "half" else (2 * i, 2 * i + 1) for i in range(half)]
    a, b = (torch.tensor([p[j] for p in first], device=DEV) for j in (0, 1))
    place = torch.cat([torch.arange(c, c + n, device=DEV) for c, n in zip(ctx, n_new)])
    pos = place[:, None] if s["positions"] is None else torch.stack([s["positions"][s["freq_axis"][i]] for i in range(half)], 1)
    # exp(i angle) as complex numbers
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), pos.double() * s["inv_freq"].double())[:, None, :]

    def turned(x):
        x = x.double()
        y = torch.complex(x[..., a], x[..., b]) * turn
        x[..., a], x[..., b] = y.real, y.imag
        return x

    pool = s["pool"].double()
    k, v = turned(s["k"]), s["v"].double()
    row = 0
    for i, (c, n) in enumerate(zip(ctx, n_new)):
        t = torch.arange(c, c + n, device=DEV)
        page = s["bt_pages"][int(s["bt_indptr"][i]) + t // PAGE].long()
        for part, x in ((0, k), (1, v)):
            for h in range(case["hkv"]):
                to = (page, part, h, t % PAGE) if case["layout"] == "hnd" else (page, part, t % PAGE, h)
                pool[to] = x[row:row + n, h]
        row += n
    return turned(s["q"]), pool


def _exact_prefix(case, s):
    cuts, prefix, n_q, tail = _prefix_sizes(case)
    if work(case)["flops"] > 8e11:
        return None
    rows, share = sum(n_q), case["hq"] // case["hkv"]
    out = torch.empty((rows, case["hq"], D), dtype=torch.float64, device=DEV)
    lse = torch.empty((rows, case["hq"]), dtype=torch.float64, device=DEV)
    starts, at = _indptr(n_q), s["bt_indptr"].tolist()
    heads_first = s["pool"] if case["layout"] == "hnd" else s["pool"].transpose(2, 3)
    for g, p in enumerate(prefix):
        members = range(cuts[g], cuts[g + 1])
        r0, r1 = starts[members[0]], starts[members[-1] + 1]
        shared = s["bt_pages"][at[members[0]]:at[members[0]] + p // PAGE].long()
        for h in range(case["hkv"]):
            qh = s["q"][r0:r1, h * share:(h + 1) * share].double() / math.sqrt(D)
            k, v = (heads_first[shared, part, h].double().reshape(-1, D) for part in (0, 1))
            z = torch.einsum("rgd,td->rgt", qh, k)
            top = z.amax(-1)
            w = (z - top[..., None]).exp()
            total, part_out = w.sum(-1), torch.einsum("rgt,td->rgd", w, v)
            del z, w
            for b in members:
                i, j = starts[b] - r0, starts[b + 1] - r0
                mine = s["bt_pages"][at[b] + p // PAGE:at[b + 1]].long()
                k, v = (heads_first[mine, part, h].double().reshape(-1, D)[:tail[b]] for part in (0, 1))
                z = torch.einsum("rgd,td->rgt", qh[i:j], k)
                seen = torch.ones(n_q[b], tail[b], dtype=torch.bool, device=DEV).tril(tail[b] - n_q[b])
                z = torch.where(seen[:, None], z, -math.inf)
                both = torch.maximum(top[i:j], z.amax(-1))
                scale, w = (top[i:j] - both).exp(), (z - both[..., None]).exp()
                sums = total[i:j] * scale + w.sum(-1)
                to = slice(h * share, (h + 1) * share)
                out[r0 + i:r0 + j, to] = (part_out[i:j] * scale[..., None] + torch.einsum("rgt,td->rgd", w, v)) / sums[..., None]
                lse[r0 + i:r0 + j, to] = both + sums.log()
    return out, lse


def _exact_sample(case, s):
    """Row by row, from the definition; the tokens are whole numbers and have no value in 64 bits of their own."""
    x, u = s["logits"].double(), s["uniform"].tolist()
    settings = {n: None if s[n] is None else s[n].tolist() for n in ("temperature", "top_k", "top_p", "min_p")}
    logprob = []
    for r in range(case["rows"]):
        row, t = x[r], settings["temperature"][r]
        if not t > 0:
            logprob.append(0.0)
            continue
        p = torch.softmax(row / t, 0)
        by_value = torch.argsort(-row, stable=True)
        k = settings["top_k"][r] if settings["top_k"] else 0
        if 0 < k < case["vocab"]:
            by_value = by_value[:k]
        share = p[by_value] / p[by_value].sum()
        q = settings["top_p"][r] if settings["top_p"] else 1.0
        if q < 1:
            by_value = by_value[:1 + int((share.cumsum(0) < q).sum())]
        if settings["min_p"] and settings["min_p"][r] > 0:
            by_value = by_value[p[by_value] >= settings["min_p"][r] * p[by_value[0]]]
        by_index = by_value.sort().values
        chance = p[by_index] / p[by_index].sum()
        logprob.append(chance[torch.searchsorted(chance.cumsum(0), u[r], right=True).clamp(max=len(chance) - 1)].log().item())
    return None, torch.tensor(logprob, dtype=torch.float64)
