"""The operators of a serving program around the compressed cache: attention of a prompt with a sliding window and
sinks, and a key-value cache in pages that is filled, attended over by one new token per sequence, and evicted from by
accumulated attention weight.

A case names one operator (`kind`) and its sizes:

  attention  d2o_prompt_attention: causal attention of a prompt, `window` keys back (0: all of them), the first `sinks`
             keys always visible; `lse`: with the row normalisers that d2o_layer_stats takes; `ragged`: every sequence
             has its own length
  append     d2o_paged_append: the keys and values of a prompt, or of a turn, go into the pages behind the rows that
             are there; `score`: with their positions and the column sums of the prompt attention, summed over the
             query heads of a key head, as scores
  decode     d2o_paged_decode_step: one new token per sequence, appended and attended with; `score`: the weights are
             added to the rows' scores
  evict      d2o_paged_evict: the rows with the lowest scores leave, what is kept ends up in the first `budget` rows

Shapes are those of the other workloads of this folder: a small fp32 stack (8 heads, d = 64), the 7B-like one (32 query
heads, 32 KV heads, d = 128, fp16) and the 8B-like one (32 / 8, d = 128, bf16).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SMALL = (8, 8, 64, "f32")
MHA = (32, 32, 128, "f16")
GQA = (32, 8, 128, "bf16")


def _shape(shape):
    q, kv, d, dtype = shape
    return dict(q_heads=q, kv_heads=kv, d_head=d, dtype=dtype)


def _attention(shape, batch, prompt, window, sinks, lse, ragged):
    return dict(kind="attention", **_shape(shape), batch=batch, prompt=prompt, window=window, sinks=sinks, lse=lse,
                ragged=ragged)


def _append(shape, batch, page, held, rows, score):
    return dict(kind="append", **_shape(shape), batch=batch, page=page, held=held, rows=rows, score=score)


def _decode(shape, batch, page, held, ragged, window, sinks, score):
    return dict(kind="decode", **_shape(shape), batch=batch, page=page, held=held, ragged=ragged, window=window,
                sinks=sinks, score=score)


def _evict(shape, batch, page, held, budget, window, sinks, evicted_before):
    return dict(kind="evict", **_shape(shape), batch=batch, page=page, held=held, budget=budget, window=window,
                sinks=sinks, evicted_before=evicted_before)


def listed():
    return [
        # a layer of a small fp32 model with a short window
        dict(_attention(SMALL, 1, 1024, 256, 4, True, False), name="attention fp32 small"),
        # a chat prompt; its normalisers go to the column sums
        dict(_attention(MHA, 1, 1200, 0, 0, True, False), name="attention 7b chat"),
        # four prompts of their users' lengths, the longest a multiple of nothing
        dict(_attention(GQA, 4, 6001, 0, 0, True, True), name="attention 8b ragged"),
        # a long document under a window, with the first tokens as sinks
        dict(_attention(GQA, 1, 32768, 4096, 4, False, False), name="attention 8b window"),
        # sixteen follow-up turns of a few tokens
        dict(_append(GQA, 16, 16, 4000, 45, False), name="append 8b turn"),
        # four prompts with the scores that the eviction goes by
        dict(_append(MHA, 4, 64, 0, 4096, True), name="append 7b prompt"),
        # one conversation: the smallest call, where latency counts
        dict(_decode(GQA, 1, 16, 1640, False, 0, 0, False), name="decode 8b single"),
        # eight conversations of any length, weights kept for the eviction
        dict(_decode(MHA, 8, 64, 4096, True, 0, 0, True), name="decode 7b scores"),
        # one long document: few slices, each of them long
        dict(_decode(GQA, 1, 64, 131072, False, 0, 0, False), name="decode 8b long"),
        # a batch of long conversations of which a window and the first tokens are seen
        dict(_decode(GQA, 32, 16, 16384, True, 2048, 4, False), name="decode 8b window"),
        # the prompt stage's eviction of a long document
        dict(_evict(GQA, 1, 64, 32768, 6554, 1638, 1, False), name="evict 8b prompt"),
        # every sixteen generated tokens the cache goes back to its size
        dict(_evict(MHA, 8, 16, 2064, 2048, 512, 4, True), name="evict 7b generation"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attention", "append", "decode", "decode", "evict"])
    shape = rng.choice([SMALL, MHA, GQA, GQA])
    q, kv, d, dtype = shape
    page = rng.choice([16, 32, 64, 128])
    # rows of one head that a case may hold: what the largest listed cases hold
    most = 131072 * 8 * 256 // (kv * d * (4 if dtype == "f32" else 2))
    if kind == "attention":
        batch = rng.choice([1, 1, 2, 4])
        prompt = _log(rng, 64, 2400 if dtype == "f32" else 6000)
        window = rng.choice([0, _log(rng, 16, prompt)])
        return _attention(shape, batch, prompt, window, rng.choice([0, 1, 4, 100]) if window else 0, rng.random() < 0.5,
                          batch > 1)
    batch = _log(rng, 1, 48)
    if kind == "append":
        rows = _log(rng, 1, max(2, min(16384, most // 2 // batch)))
        return _append(shape, batch, page, rng.choice([0, _log(rng, 1, 4096)]), rows, rng.random() < 0.5)
    if kind == "decode":
        held = _log(rng, 1, min(131071, most // 2 // batch))
        window = rng.choice([0, 0, _log(rng, 16, 8192)])
        return _decode(shape, batch, page, held, batch > 1, window, rng.choice([0, 4]) if window else 0, rng.random() < 0.4)
    held = _log(rng, 24, min(32768, most // 2 // batch))
    budget = max(8, int(held * rng.uniform(0.1, 1.0)))
    return _evict(shape, batch, page, held, budget, budget // 4, rng.choice([0, 1, 4]), rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _keys(g, b, h, n, d):
    """Keys of a few directions with noise around them; the first is a sink that the queries of _queries look at."""
    z = torch.randn(b, h, n, 8, generator=g, device=DEV)
    w = torch.randn(1, h, 8, d, generator=g, device=DEV) / math.sqrt(8)
    k = torch.matmul(z, w).add_(torch.randn(b, h, n, d, generator=g, device=DEV), alpha=0.3)
    return k, w


def _queries(g, b, hq, n, d, w):
    """Queries along the directions of their key head, so that the weights are neither flat nor on one key."""
    z = torch.randn(b, hq, n, 8, generator=g, device=DEV) * 0.8
    w = w.repeat_interleave(hq // w.shape[1], dim=1)
    return torch.matmul(z, w).add_(torch.randn(b, hq, n, d, generator=g, device=DEV), alpha=0.5)


def _lengths(g, case, n, least=1):
    """Lengths of a ragged batch: the first is the longest, the others are spread down to a tenth of it."""
    if not case.get("ragged"):
        return torch.full((case["batch"],), n, dtype=torch.int32, device=DEV)
    f = torch.exp(-2.3 * torch.rand(case["batch"], generator=g, device=DEV, dtype=torch.float64))
    f[0] = 1.0
    return (f * n).round().clamp(min=least).to(torch.int32)


def _pages(g, case, rows):
    """A page table for up to `rows` rows of every sequence, pages in the order in which an allocator handed them out."""
    per = -(-rows // case["page"])
    n = per * case["batch"] + 3
    table = torch.randperm(n, generator=g, device=DEV)[: per * case["batch"]].to(torch.int32)
    return n, table.view(case["batch"], per)


def prepare(case, seed):
    g, dt, dev = _gen(seed), DTYPE[case["dtype"]], DEV
    b, hq, h, d = case["batch"], case["q_heads"], case["kv_heads"], case["d_head"]
    s = dict(case=case)
    if case["kind"] == "attention":
        n = case["prompt"]
        k, w = _keys(g, b, h, n, d)
        s["q"], s["k"] = _queries(g, b, hq, n, d, w).to(dt), k.to(dt)
        s["v"] = torch.randn(b, h, n, d, generator=g, device=dev).to(dt)
        s["lens"] = _lengths(g, case, n) if case["ragged"] else None
        s["out"] = torch.zeros(b, hq, n, d, dtype=dt, device=dev)
        s["lse"] = torch.zeros(b, hq, n, dtype=torch.float32, device=dev) if case["lse"] else None
        return s
    page = case["page"]
    held = _lengths(g, case, case["held"])
    n_rows = case["held"] + {"append": case.get("rows", 0), "decode": 1, "evict": 0}[case["kind"]]
    n_pages, s["table"] = _pages(g, case, n_rows)
    s["len"] = held[:, None].expand(b, h).contiguous()
    shape = (n_pages, h, page)
    scored = case["kind"] == "evict" or case["score"]
    # positions and scores lie in one buffer, which the eviction's cases restore in one copy
    s["rows"] = torch.zeros(2, *shape, dtype=torch.int32, device=dev) if scored else None
    s["pos"] = s["rows"][0] if scored else None
    s["score"] = s["rows"][1].view(torch.float32) if scored else None
    k, w = _keys(g, n_pages, h, page, d)
    s["k_pages"] = k.to(dt)
    s["v_pages"] = torch.randn(*shape, d, generator=g, device=dev).to(dt)
    del k
    if case["kind"] == "append":
        n = case["rows"]
        s["k"] = _keys(g, b, h, n, d)[0].to(dt)
        s["v"] = torch.randn(b, h, n, d, generator=g, device=dev).to(dt)
        lens = (n * torch.rand(b, generator=g, device=dev, dtype=torch.float64)).ceil()
        s["lens"] = None if case["score"] else lens.clamp(1, n).to(torch.int32)
        s["first"] = held.clone() if scored else None
        s["colsum"] = torch.rand(b, hq, n, generator=g, device=dev).mul_(4).exp_() if scored else None
    elif case["kind"] == "decode":
        s["q"] = _queries(g, b, hq, 1, d, w)[:, :, 0].to(dt)
        s["nk"] = (torch.matmul(torch.randn(b, h, 1, 8, generator=g, device=dev), w)[:, :, 0]).to(dt)
        s["nv"] = torch.randn(b, h, d, generator=g, device=dev).to(dt)
        s["out"] = torch.zeros(b, hq, d, dtype=dt, device=dev)
        s["positions"] = held.clone() if scored else None
        if scored:
            s["score"].copy_(torch.randn(*shape, generator=g, device=dev).exp_())
            s["pos"].copy_(torch.randint(0, 1 << 20, shape, generator=g, device=dev))
    else:
        # scores as a model hands them over in 16 bits: some are equal
        s["score"].copy_((torch.randn(*shape, generator=g, device=dev) * 2).exp_().half().float())
        n, cap = case["held"], s["table"].shape[1] * page
        seen = n + (n // 2 if case["evicted_before"] else 0)
        if case["evicted_before"]:      # a subset of the positions, in the order that earlier evictions left
            at = torch.rand(b, h, seen, generator=g, device=dev).argsort(-1)[..., :n]
        else:
            at = torch.arange(n, device=dev).expand(b, h, n)
        at = torch.nn.functional.pad(at, (0, cap - n)).to(torch.int32)
        s["pos"][s["table"].long()] = at.view(b, h, -1, page).transpose(1, 2)
        s["rows0"] = s["rows"].clone()
        s["budgets"] = torch.full((b, h), case["budget"], dtype=torch.int32, device=dev)
        s["next"] = torch.full((b,), seen, dtype=torch.int32, device=dev)
    if own:
        from paper_2406_13035_b200 import binding
        s["cache"] = binding.D2OPagedCache(s["k_pages"], s["v_pages"], s["table"], s["len"], n_q_heads=hq, pos=s["pos"],
                                           score=s["score"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _visible(rows, cols, window, sinks):
    m = cols <= rows
    return m & ((cols > rows - window) | (cols < sinks)) if window else m


def _plain_attention(s):
    c = s["case"]
    b, hq, h, d, n = c["batch"], c["q_heads"], c["kv_heads"], c["d_head"], c["prompt"]
    q = s["q"].view(b, h, hq // h, n, d)
    at = torch.arange(n, device=DEV)
    block = max(64, min(n, (1 << 28) // (b * hq * n)))          # queries at a time: the weights of all would not fit
    for r0 in range(0, n, block):
        r1 = min(n, r0 + block)
        lo = max(0, r0 - c["window"] + 1) if c["window"] else 0
        cols = torch.cat([at[: min(lo, c["sinks"])], at[lo:r1]])
        k, v = s["k"][:, :, cols].float(), s["v"][:, :, cols].float()
        x = torch.matmul(q[:, :, :, r0:r1].float().flatten(2, 3), k.transpose(2, 3)).view(b, h, hq // h, r1 - r0, -1)
        x = (x / math.sqrt(d)).masked_fill(~_visible(at[r0:r1, None], cols, c["window"], c["sinks"]), -math.inf)
        top = x.amax(-1, keepdim=True)
        p = torch.exp(x - top)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul((p / total).flatten(2, 3), v).view(b, hq, r1 - r0, d)
        lse = (top + torch.log(total)).view(b, hq, r1 - r0)
        if s["lens"] is not None:                               # rows behind a sequence's end stay as they were
            live = (at[r0:r1] < s["lens"][:, None])[:, None]
            o = torch.where(live[..., None], o, s["out"][:, :, r0:r1].float())
            lse = torch.where(live, lse, s["lse"][:, :, r0:r1]) if s["lse"] is not None else lse
        s["out"][:, :, r0:r1] = o.to(s["out"].dtype)
        if s["lse"] is not None:
            s["lse"][:, :, r0:r1] = lse
    return {"out": s["out"], "lse": s["lse"]}


def _plain_append(s):
    c = s["case"]
    b, h, n, page = c["batch"], c["kv_heads"], c["rows"], c["page"]
    i = torch.arange(n, device=DEV).expand(b, n)
    live = i < s["lens"][:, None] if s["lens"] is not None else torch.ones_like(i, dtype=torch.bool)
    seq, i = live.nonzero(as_tuple=True)
    slot = s["len"][seq, 0] + i
    pg, at = s["table"][seq, slot // page].long(), slot % page
    s["k_pages"][pg, :, at] = s["k"][seq, :, i]
    s["v_pages"][pg, :, at] = s["v"][seq, :, i]
    if s["pos"] is not None:
        s["pos"][pg, :, at] = (s["first"][seq] + i).to(torch.int32)[:, None].expand(-1, h)
        s["score"][pg, :, at] = s["colsum"].view(b, h, -1, n).sum(2)[seq, :, i]
    return {"k": s["k_pages"], "v": s["v_pages"], "pos": s["pos"], "score": s["score"]}


def _plain_decode(s, t=torch.float32):
    c = s["case"]
    b, hq, h, d, page = c["batch"], c["q_heads"], c["kv_heads"], c["d_head"], c["page"]
    seq, n = torch.arange(b, device=DEV), s["len"][:, 0]
    pg, at = s["table"][seq, n // page].long(), n % page
    s["k_pages"][pg, :, at], s["v_pages"][pg, :, at] = s["nk"], s["nv"]
    table = s["table"].long()

    def dense(pages):                                           # [B, Hkv, rows, ...] of what the table reaches
        return pages[table].transpose(1, 2).flatten(2, 3)

    slot = torch.arange(table.shape[1] * page, device=DEV)
    seen = _visible(n[:, None], slot, c["window"], c["sinks"])[:, None, None]
    x = torch.matmul(s["q"].view(b, h, -1, d).to(t), dense(s["k_pages"]).to(t).transpose(2, 3)) / math.sqrt(d)
    x = x.masked_fill(~seen, -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    p = p / p.sum(-1, keepdim=True)
    s["out"].copy_(torch.matmul(p, dense(s["v_pages"]).to(t)).view(b, hq, d))
    if s["score"] is not None:
        s["pos"][pg, :, at] = s["positions"][:, None].expand(-1, h)
        s["score"][pg, :, at] = 0.0
        s["score"].index_add_(0, table.flatten(), p.sum(2).view(b, h, -1, page).transpose(1, 2).flatten(0, 1).float())
    return {"out": s["out"], "k": s["k_pages"], "v": s["v_pages"], "pos": s["pos"], "score": s["score"]}


def _plain_evict(s):
    c = s["case"]
    b, h, page = c["batch"], c["kv_heads"], c["page"]
    table = s["table"].long()

    def dense(pages):
        return pages[table].transpose(1, 2).flatten(2, 3)

    pos, score = dense(s["pos"]), dense(s["score"])
    slot = torch.arange(pos.shape[-1], device=DEV).expand_as(pos)
    n = s["len"][..., None]
    budget = torch.minimum(s["budgets"][..., None], n)
    held = slot < n
    sure = held & ((pos < c["sinks"]) | (pos >= s["next"][:, None, None] - c["window"]))
    # highest first, protected rows ahead of all, rows that are not there behind all; ties by position
    order = torch.where(held, pos, 1 << 30).sort(dim=-1, stable=True).indices
    key = score.masked_fill(sure, math.inf).masked_fill(~held, -math.inf)
    order = order.gather(-1, key.gather(-1, order).sort(dim=-1, descending=True, stable=True).indices)
    rank = torch.empty_like(order).scatter_(-1, order, slot)
    kept = rank < budget
    to, frm = (slot < budget) & ~kept, (slot >= budget) & kept
    bi, hi, ti = to.nonzero(as_tuple=True)                      # both ascend, with as many of each in every slice
    _, _, fi = frm.nonzero(as_tuple=True)
    tp, fp = table[bi, ti // page], table[bi, fi // page]
    for a in (s["k_pages"], s["v_pages"], s["pos"], s["score"]):
        a[tp, hi, ti % page] = a[fp, hi, fi % page]
    return {"k": s["k_pages"], "v": s["v_pages"], "pos": s["pos"], "score": s["score"]}


def run(s):
    c = s["case"]
    if c["kind"] == "evict":
        s["rows"].copy_(s["rows0"])         # the eviction works in place: without this a second pass would find nothing to do
    if not own:
        return {"attention": _plain_attention, "append": _plain_append, "decode": _plain_decode, "evict": _plain_evict}[c["kind"]](s)
    from paper_2406_13035_b200 import binding
    if c["kind"] == "attention":
        binding.d2o_prompt_attention(s["q"], s["k"], s["v"], s["out"], lse=s["lse"], window=c["window"], n_sink=c["sinks"],
                                     lens=s["lens"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["kind"] == "append":
        s["cache"].d2o_paged_append(s["k"], s["v"], lens=s["lens"], first_pos=s["first"], colsum=s["colsum"])
    elif c["kind"] == "decode":
        s["cache"].d2o_paged_decode_step(s["q"], s["nk"], s["nv"], s["out"], positions=s["positions"], window=c["window"],
                                         n_sink=c["sinks"])
    else:
        s["cache"].d2o_paged_evict(s["budgets"], s["next"], window=c["window"], n_sink=c["sinks"])
    got = {"k": s["k_pages"], "v": s["v_pages"], "pos": s["pos"], "score": s["score"]}
    return dict(out=s["out"], **got) if c["kind"] == "decode" else got


# ------------------------------------------------------------------------------------------------ work
def _mean_length(case, n):
    """Of _lengths: one sequence of n, the others n * exp(-2.3 u)."""
    if not case.get("ragged"):
        return float(n)
    return n * (1 + (case["batch"] - 1) * (1 - math.exp(-2.3)) / 2.3) / case["batch"]


def work(case):
    b, hq, h, d = case["batch"], case["q_heads"], case["kv_heads"], case["d_head"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "attention":
        n, w = case["prompt"], case["window"] or case["prompt"]
        lens = [n] if not case["ragged"] else [n] + [n * math.exp(-2.3 * (i + 0.5) / max(1, b - 1)) for i in range(b - 1)]
        pairs = sum(m * (m + 1) / 2 - max(0.0, m - w) * (m - w + 1) / 2 + case["sinks"] * max(0.0, m - w - case["sinks"] / 2)
                    for m in lens) * (1 if case["ragged"] else b)
        rows = sum(lens) * (1 if case["ragged"] else b)
        return {"bytes": rows * (d * e * (2 * hq + 2 * h) + (4 * hq if case["lse"] else 0)), "flops": 4.0 * d * pairs * hq}
    row = 2 * d * e
    if case["kind"] == "append":
        n = case["rows"] if case["score"] else (case["rows"] + 1) / 2
        return {"bytes": b * n * (2 * row * h + (4 * hq + 8 * h if case["score"] else 0)), "flops": 0}
    if case["kind"] == "decode":
        m = _mean_length(case, case["held"]) + 1
        if case["window"]:
            m = min(m, case["window"] + case["sinks"])
        return {"bytes": b * h * m * (row + (8 if case["score"] else 0)) + b * (hq * 2 * d * e + h * 2 * row),
                "flops": 4.0 * d * b * hq * m}
    n, k = case["held"], min(case["budget"], case["held"])
    moved = k * (n - k) / n if not case["window"] else max(0.0, k - case["sinks"]) * (1 - (k - case["window"]) / max(1, n - case["window"]))
    moved = min(moved, n - k)
    return {"bytes": b * h * (8 * n + moved * (2 * row + 16)), "flops": 0}


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    b, hq, h, d = case["batch"], case["q_heads"], case["kv_heads"], case["d_head"]
    group = hq // h
    if case["kind"] == "attention":
        n, w, t = case["prompt"], case["window"] or case["prompt"], case["sinks"]
        out, lse = s["out"].double(), None if s["lse"] is None else s["lse"].double()
        for i in range(b):
            m = n if s["lens"] is None else int(s["lens"][i])
            for x in range(hq):
                q, k, v = (y.double() for y in (s["q"][i, x, :m], s["k"][i, x // group, :m], s["v"][i, x // group, :m]))
                for r0 in range(0, m, 4096):
                    r1 = min(m, r0 + 4096)
                    lo = max(0, r0 - w + 1)
                    lo = 0 if lo <= t else lo
                    z = q[r0:r1] @ k[lo:r1].T / math.sqrt(d)
                    r, j = torch.arange(r0, r1, device=DEV)[:, None], torch.arange(lo, r1, device=DEV)[None]
                    z = torch.where((j <= r) & ((r - j < w) | (j < t)), z, -math.inf)
                    if lo:
                        z = torch.cat([q[r0:r1] @ k[:t].T / math.sqrt(d), z], 1)
                    y = torch.logsumexp(z, 1)
                    a = torch.exp(z - y[:, None])
                    out[i, x, r0:r1] = a[:, a.shape[1] - (r1 - lo):] @ v[lo:r1] + (a[:, :t] @ v[:t] if lo else 0.0)
                    if lse is not None:
                        lse[i, x, r0:r1] = y
        return {"out": out, "lse": lse}
    if case["kind"] == "append":
        if s["score"] is None:
            return None
        score = s["score"].double()
        sums = sum(s["colsum"].double().view(b, h, group, -1)[:, :, j] for j in range(group))
        for i in range(b):
            slots = s["len"][i, 0] + torch.arange(case["rows"], device=DEV)
            score[s["table"][i].long()[slots // case["page"]], :, slots % case["page"]] = sums[i].T
        return {"k": None, "v": None, "pos": None, "score": score}
    if case["kind"] == "decode":
        out = torch.zeros(b, hq, d, dtype=torch.float64, device=DEV)
        score = None if s["score"] is None else s["score"].double()
        for i in range(b):
            n = int(s["len"][i, 0])
            slots = torch.arange(n, device=DEV)
            if case["window"]:
                slots = slots[(slots > n - case["window"]) | (slots < case["sinks"])]
            pg, at = s["table"][i].long()[slots // case["page"]], slots % case["page"]
            k = torch.cat([s["k_pages"][pg, :, at].double(), s["nk"][i][None].double()])       # [rows, Hkv, d]
            v = torch.cat([s["v_pages"][pg, :, at].double(), s["nv"][i][None].double()])
            z = torch.einsum("hgd,nhd->hgn", s["q"][i].double().view(h, group, d), k) / math.sqrt(d)
            a = torch.softmax(z, -1)
            out[i] = torch.einsum("hgn,nhd->hgd", a, v).reshape(hq, d)
            if score is not None:
                weight = a.sum(1).T                                                             # [rows, Hkv]
                score[pg, :, at] += weight[:-1]
                score[int(s["table"][i, n // case["page"]]), :, n % case["page"]] = weight[-1]
        return {"out": out, "k": None, "v": None, "pos": None, "score": score}
    return None
