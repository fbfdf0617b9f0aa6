"""Cases, plain forms and calls of the operators around a paged KV cache: rows appended to it, attention of chunks of new
tokens over it, the attention weight that each of its rows gathers, eviction by that weight; and log probabilities of given tokens.

A paged cache of n_seq sequences: k, v [n_pages, page_size, Hkv, d], pos and weight [n_pages, page_size], a table
[n_seq, max_pages] of page numbers and len [n_seq].  Row j of sequence b lies in page table[b, j // page_size] at j % page_size.
The queries of a call are the last rows of their sequences: query i of n sees rows j <= len - n + i.
"""
import math

import torch

own = False

LLAMA = {"heads": 32, "kv_heads": 8, "dim": 128}
QWEN = {"heads": 28, "kv_heads": 4, "dim": 128}
TINY = {"heads": 4, "kv_heads": 2, "dim": 64}


def listed():
    return [
        # one decode step of a running batch: one new row per sequence
        {"name": "append_64x1", "op": "append", **LLAMA, "n_seq": 64, "rows": 1, "longest": 8192, "page": 64, "dtype": "bf16"},
        # packed chunks of prompts of different lengths enter the cache, small pages
        {"name": "append_8_chunks", "op": "append", **LLAMA, "n_seq": 8, "rows": 4099, "longest": 16384, "page": 16, "dtype": "bf16"},
        # one token over a short context: latency counts
        {"name": "attention_1x777", "op": "attention", **LLAMA, "n_seq": 1, "rows": 1, "longest": 777, "page": 64, "dtype": "bf16"},
        # a running batch that verifies up to nine drafted tokens a sequence, an odd number of query heads per KV head, small
        # pages, one sequence that takes part with no token and one whose cache is empty
        {"name": "attention_48_drafts", "op": "attention", **QWEN, "n_seq": 48, "rows": 9, "longest": 16384, "page": 16, "dtype": "bf16"},
        # the next turn of a conversation: a long chunk over a long context
        {"name": "attention_chunk_2048", "op": "attention", **LLAMA, "n_seq": 1, "rows": 2048, "longest": 34816, "page": 64, "dtype": "bf16"},
        # fp32 storage, the small head size, ragged short chunks
        {"name": "attention_fp32_3x37", "op": "attention", **TINY, "n_seq": 3, "rows": 37, "longest": 1000, "page": 32, "dtype": "fp32"},
        # a decode step of a batch notes what its tokens looked at
        {"name": "weights_16x1", "op": "weights", **LLAMA, "n_seq": 16, "rows": 1, "longest": 8192, "page": 64, "dtype": "bf16"},
        # the last 64 tokens of a long prompt judge its rows before the cache is cut down
        {"name": "weights_window_64", "op": "weights", **LLAMA, "n_seq": 1, "rows": 64, "longest": 32768, "page": 128, "dtype": "bf16"},
        # the cache of a long prompt is cut down once
        {"name": "evict_32768", "op": "evict", **LLAMA, "n_seq": 1, "longest": 32768, "keep": 4096, "sink": 4, "recent": 256, "page": 64, "dtype": "bf16"},
        # a batch at its budget: every sequence gives up the few rows that it grew by
        {"name": "evict_48_ragged", "op": "evict", **QWEN, "n_seq": 48, "longest": 4111, "keep": 4096, "sink": 4, "recent": 64, "page": 16, "dtype": "bf16"},
        # the token that a decode step chose, with five alternatives: latency counts
        {"name": "logprobs_1x128256", "op": "logprobs", "n": 1, "vocab": 128256, "top": 5},
        # a chunk of a prompt is scored, odd vocabulary
        {"name": "logprobs_509x152063", "op": "logprobs", "n": 509, "vocab": 152063, "top": 20},
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "weights", "evict", "logprobs"])
    if op == "logprobs":
        n = _spread(rng, 1, 512)
        return {"op": op, "n": n, "vocab": _spread(rng, 100, 152064), "top": rng.choice([0, 1, 5, 20, 32])}
    dtype = "fp32" if rng.random() < 0.15 else "bf16"
    kv = rng.choice([1, 2, 4, 8])
    case = {"op": op, "heads": kv * rng.choice([1, 2, 4, 7, 8]), "kv_heads": kv, "dim": rng.choice([64, 128, 128]), "n_seq": _spread(rng, 1, 64),
            "page": rng.choice([16, 32, 64, 128, 256]), "dtype": dtype}
    case["longest"] = longest = _spread(rng, 16, min(32768, 262144 // case["n_seq"]) if dtype == "bf16" else 4096)
    if op == "evict":
        case["keep"] = rng.randrange(1, longest + 1)
        case["sink"], case["recent"] = rng.choice([0, 4, 16]), rng.choice([0, 1, 64, 512])
        return case
    rows = 1 if rng.random() < 0.3 else _spread(rng, 1, longest)
    if op != "append":
        # no more pairs of a query and a row than in the listed chunk
        most = (1 << 31) if dtype == "bf16" else (1 << 27)
        rows = max(1, min(rows, most // (case["heads"] * longest * case["n_seq"])))
    case["rows"] = rows
    return case


def _ragged(case):
    """Rows held and rows of the call for each sequence: lengths from a few rows to the longest, one sequence with nothing held and
    one with nothing in the call where there are several."""
    n, longest, most = case["n_seq"], case["longest"], case.get("rows", 0)
    lens = [max(1, round(longest * ((i + 1) / n) ** 1.5)) for i in range(n)]
    if case["op"] == "evict":
        lens = [max(1, round(longest * (0.9 + 0.1 * (i + 1) / n))) for i in range(n)]
    if n > 2 and case["op"] != "append":
        lens[n // 2] = 0
    if most <= 1:
        return lens, [min(1, most)] * n
    # chunks of all sizes, long ones also for short contexts
    rows = [1 + (most - 1) * (7 * i % n) // max(1, n - 1) for i in range(n)]
    rows[n - 1] = most
    rows = [min(r, held) if held else r for r, held in zip(rows, lens)]
    if n > 2:
        rows[n // 3] = 0
    return lens, rows


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _context(case):
    from paper_2601_13155_b200 import binding, synth

    heads, kv_heads, dim = (case["heads"], case["kv_heads"], case["dim"]) if "heads" in case else (4, 2, 64)
    shape = synth.ModelShape(hidden=heads * dim, n_q_heads=heads, n_kv_heads=kv_heads, head_dim=dim, ffn_dim=256, ltp_dlow=64, ltp_rank=16,
                             n_layers=1, vocab=64, dtype=case.get("dtype", "bf16"))
    return binding.Spts(shape, max_seq=64), shape


def prepare(case, seed):
    gen = _generator(seed)
    st = {"case": case}
    if case["op"] == "logprobs":
        n, v = case["n"], case["vocab"]
        st["logits"] = 3.0 * torch.randn(n, v, device="cuda", generator=gen)
        # most tokens that are scored are likely ones; a row in three has a grammar that forbids every second token
        likely = torch.topk(st["logits"], min(v, 8), -1).indices
        pick = torch.randint(0, likely.shape[1], (n, 1), device="cuda", generator=gen)
        other = torch.randint(0, v, (n,), device="cuda", generator=gen)
        st["targets"] = torch.where(torch.rand(n, device="cuda", generator=gen) < 0.8, likely.gather(1, pick)[:, 0], other).to(torch.int32)
        st["logits"][1::3, 1::2] = float("-inf")
        if own:
            st["lib"], _ = _context(case)
        return st
    n, hkv, d, page, longest = case["n_seq"], case["kv_heads"], case["dim"], case["page"], case["longest"]
    dt = _type(case)
    # a ragged batch: the same lengths and chunks in another order for each seed
    lens, rows = _ragged(case)
    mix = torch.randperm(n, device="cuda", generator=gen)
    lens, rows = torch.tensor(lens, device="cuda")[mix], torch.tensor(rows, device="cuda")[mix]
    if case["op"] != "evict":
        if case["op"] == "append":
            st["at"] = (lens - rows).to(torch.int32)
        start = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
        start[1:] = torch.cumsum(rows, 0)
        st["row_start"] = start.to(torch.int32) if case["rows"] > 1 else None
        total = int(start[-1])
    # pages in the order in which a running server hands them out
    cap = int(lens.max()) + page
    most = -(-cap // page)
    held = torch.arange(most, device="cuda")[None, :] * page < lens[:, None]
    n_pages = int(held.sum()) + 5
    st["table"] = torch.full((n, most), -1, dtype=torch.int32, device="cuda")
    st["table"][held] = torch.randperm(n_pages, device="cuda", generator=gen)[: n_pages - 5].to(torch.int32)
    st["len"] = lens.to(torch.int32)
    for name in ("k", "v"):
        st[name] = torch.randn(n_pages, page, hkv, d, device="cuda", generator=gen).to(dt)
    st["pos"] = torch.zeros(n_pages, page, dtype=torch.int32, device="cuda")
    st["weight"] = torch.zeros(n_pages, page, device="cuda")
    place = torch.arange(most * page, device="cuda")[None, :].expand(n, -1)
    inside = place < lens[:, None]
    at = _slots(st, place)[inside]
    if case["op"] == "append":
        st["k_rows"] = torch.randn(total, hkv, d, device="cuda", generator=gen).to(dt)
        st["v_rows"] = torch.randn(total, hkv, d, device="cuda", generator=gen).to(dt)
        st["pos_rows"] = torch.randint(0, 1 << 20, (total,), dtype=torch.int32, device="cuda", generator=gen)
    elif case["op"] == "evict":
        # a prefill that skipped tokens left rows of every second or third position; few rows have most of the weight
        gap = torch.randint(1, 4, (n, most * page), device="cuda", generator=gen)
        st["pos"].view(-1)[at] = torch.cumsum(gap, 1).to(torch.int32)[inside] - 1
        u = torch.rand(n, most * page, device="cuda", generator=gen)
        st["weight"].view(-1)[at] = (0.02 / (u + 1e-3))[inside]
        st["keep"] = torch.full((n,), case["keep"], dtype=torch.int32, device="cuda")
        # what changes is put back before each pass, in one copy
        slots = n_pages * page
        st["now"] = torch.cat([st["weight"].view(-1).view(torch.int32), st["pos"].view(-1), st["len"]])
        st["before"] = st["now"].clone()
        st["weight"] = st["now"][:slots].view(torch.float32).view(n_pages, page)
        st["pos"] = st["now"][slots:2 * slots].view(n_pages, page)
        st["len"] = st["now"][2 * slots:]
    else:
        # nothing has been written behind a sequence's end
        unused = torch.ones(n_pages * page, dtype=torch.bool, device="cuda")
        unused[at] = False
        for name in ("k", "v"):
            st[name].view(n_pages * page, hkv, d).masked_fill_(unused[:, None, None], float("nan"))
        st["q"] = torch.randn(total, case["heads"], d, device="cuda", generator=gen).to(dt)
        st["most_rows"] = max(_ragged(case)[1])
        if case["op"] == "weights":
            st["lse"] = _attend(st, "lse")
    if own:
        from paper_2601_13155_b200 import binding

        st["lib"], shape = _context(case)
        st["cache"] = binding.PagedKv(shape, st["table"], page_size=page, k=st["k"], v=st["v"], pos=st["pos"], weight=st["weight"], length=st["len"])
    return st


def run(state):
    return {"append": _append, "attention": _attention, "weights": _weights, "evict": _evict, "logprobs": _logprobs}[state["case"]["op"]](state)


def _slots(st, place):
    """Where rows place[b, i] of sequence b lie in the pages, counted in rows; rows in no page: slot 0."""
    page = st["case"]["page"]
    number = torch.gather(st["table"].to(torch.int64), 1, place // page)
    return number.clamp(min=0) * page + place % page


def _rows_of(st):
    """Row of the packed queries [n, most] of each sequence, and whether there is one."""
    n = st["case"]["n_seq"]
    if st["row_start"] is None:
        return torch.arange(n, device="cuda")[:, None], torch.ones(n, 1, dtype=torch.bool, device="cuda")
    start = st["row_start"].to(torch.int64)
    i = torch.arange(st["most_rows"], device="cuda")[None, :]
    there = i < (start[1:] - start[:-1])[:, None]
    return torch.where(there, start[:-1, None] + i, 0), there


def _append(st):
    case = st["case"]
    out = {"k": st["k"], "v": st["v"], "pos": st["pos"], "weight": st["weight"], "len": st["len"]}
    if own:
        st["lib"].paged_append(st["cache"], st["k_rows"], st["v_rows"], pos=st["pos_rows"], row_start=st["row_start"], at=st["at"])
        return out
    n, total = case["n_seq"], st["k_rows"].shape[0]
    start = torch.arange(n + 1, device="cuda") if st["row_start"] is None else st["row_start"].to(torch.int64)
    row = torch.arange(total, device="cuda")
    seq = torch.searchsorted(start[1:].contiguous(), row, right=True)
    j = st["at"].to(torch.int64)[seq] + row - start[seq]
    slot = st["table"].to(torch.int64)[seq, j // case["page"]] * case["page"] + j % case["page"]
    for name in ("k", "v"):
        st[name].view(-1, *st[name].shape[2:])[slot] = st[name + "_rows"]
    st["pos"].view(-1)[slot] = st["pos_rows"]
    st["weight"].view(-1)[slot] = 0.0
    st["len"].copy_((st["at"].to(torch.int64) + start[1:] - start[:-1]).to(torch.int32))
    return out


def _attend(st, want):
    """"out": attention and the log of the sum of its exponentials; "lse": that alone; "weights": the weight that every row [n, cap] gets."""
    case, q = st["case"], st["q"]
    n, h, hkv, d = case["n_seq"], case["heads"], case["kv_heads"], case["dim"]
    lens = st["len"].to(torch.int64)
    row, there = _rows_of(st)
    count = there.sum(1)
    place = torch.arange(st["table"].shape[1] * case["page"], device="cuda")
    place = place[None, : case["longest"]].expand(n, -1)
    slot = _slots(st, place)
    held = place < lens[:, None]
    k = st["k"].view(-1, hkv, d)[slot].to(torch.float32).permute(0, 2, 1, 3)                       # [n, hkv, cap, d]
    m = row.shape[1]
    qf = q.to(torch.float32)[row].view(n, m, hkv, h // hkv, d).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, d)
    s = (qf @ k.transpose(-1, -2)).view(n, hkv, h // hkv, m, -1) / math.sqrt(d)
    last = (lens - count)[:, None] + torch.arange(m, device="cuda")[None, :]
    seen = held[:, None, :] & (place[:, None, :] <= last[:, :, None]) & there[:, :, None]              # [n, m, cap]
    s = torch.where(seen[:, None, None], s, float("-inf"))
    if want == "weights":
        lse = st["lse"].to(torch.float32)[row].view(n, m, hkv, h // hkv).permute(0, 2, 3, 1)
        p = torch.exp(s - torch.where(lse == float("-inf"), 0.0, lse)[..., None])
        return p.sum((1, 2, 3)) / h, slot, held
    top = s.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), 0.0, top)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    lse = torch.zeros(q.shape[0], h, device="cuda")
    lse[row[there]] = (top + torch.log(total))[..., 0].permute(0, 3, 1, 2).reshape(n, m, h)[there]
    if want == "lse":
        return lse
    v = torch.where(held[..., None, None], st["v"].view(-1, hkv, d)[slot].to(torch.float32), 0.0).permute(0, 2, 1, 3)
    o = (p.view(n, hkv, -1, p.shape[-1]) @ v).view(n, hkv, h // hkv, m, d) / total.clamp(min=1e-30)
    out = torch.zeros(q.shape[0], h * d, dtype=q.dtype, device="cuda")
    out[row[there]] = o.permute(0, 3, 1, 2, 4).reshape(n, m, h * d)[there].to(q.dtype)
    return {"out": out, "lse": lse}


def _attention(st):
    if own:
        out, lse = st["lib"].paged_attention(st["cache"], st["q"], row_start=st["row_start"], want_lse=True)
        return {"out": out, "lse": lse}
    return _attend(st, "out")


def _weights(st):
    if own:
        st["lib"].paged_weights(st["cache"], st["q"], st["lse"], row_start=st["row_start"], decay=0.0)
        return st["weight"]
    new, slot, held = _attend(st, "weights")
    st["weight"].view(-1)[slot[held]] = new[held]
    return st["weight"]


def _evict(st):
    case = st["case"]
    st["now"].copy_(st["before"])
    out = {"k": st["k"], "v": st["v"], "pos": st["pos"], "weight": st["weight"], "len": st["len"]}
    if own:
        st["lib"].paged_evict(st["cache"], st["keep"], n_sink=case["sink"], n_recent=case["recent"])
        return out
    n, hkv, d = case["n_seq"], case["kv_heads"], case["dim"]
    lens, keep = st["len"].to(torch.int64), torch.minimum(st["keep"], st["len"]).to(torch.int64)
    place = torch.arange(case["longest"], device="cuda")[None, :].expand(n, -1)
    slot = _slots(st, place)
    held = place < lens[:, None]
    pos = st["pos"].view(-1)[slot].to(torch.int64)
    newest = torch.where(held, pos, -(1 << 40)).amax(1, keepdim=True)
    safe = (pos < case["sink"]) | (pos > newest - case["recent"])
    w = torch.where(held, torch.where(safe, float("inf"), st["weight"].view(-1)[slot]), float("-inf"))
    ranked = torch.argsort(w, dim=1, descending=True, stable=True)
    rank = torch.empty_like(ranked).scatter_(1, ranked, place.contiguous())
    stays = held & (rank < keep[:, None])
    hole = held & ~stays & (place < keep[:, None])
    mover = stays & (place >= keep[:, None])
    # the holes of a sequence, in order, take its movers, in order: there are as many of both
    src, dst = slot[mover], slot[hole]
    for t in (st["k"].view(-1, hkv, d), st["v"].view(-1, hkv, d), st["pos"].view(-1), st["weight"].view(-1)):
        t[dst] = t[src]
    st["len"].copy_(keep.to(torch.int32))
    return out


def _logprobs(st):
    case, x = st["case"], st["logits"]
    if own:
        return st["lib"].token_logprobs(x, st["targets"], n_top=case["top"])
    t = st["targets"].to(torch.int64)[:, None]
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    lse = top + torch.log(total)
    xt = x.gather(1, t)
    p = e / total
    before = (x > xt) | ((x == xt) & (torch.arange(case["vocab"], device="cuda")[None, :] < t))
    out = {"logprob": (xt - lse)[:, 0], "rank": before.sum(-1).to(torch.int32),
           "entropy": lse[:, 0] - (p * torch.where(p > 0, x, 0.0)).sum(-1)}
    if case["top"]:
        best, token = torch.sort(x, dim=-1, descending=True, stable=True)
        best, token = best[:, : case["top"]], token[:, : case["top"]].to(torch.int32)
        out["top_logprob"] = best - lse
        out["top_token"] = torch.where(best == float("-inf"), -1, token)
    return out


def work(case):
    """Bytes and operations of one pass that no way of computing it can do without."""
    op = case["op"]
    if op == "logprobs":
        n, v = case["n"], case["vocab"]
        return {"bytes": n * (4 * v + 16 + 8 * case["top"]), "flops": 6.0 * n * v}
    n, h, hkv, d = case["n_seq"], case["heads"], case["kv_heads"], case["dim"]
    e = 2 if case["dtype"] == "bf16" else 4
    row = hkv * d * e
    lens, new = _ragged(case)
    if op == "evict":
        # every row's weight and position, and the rows that move
        moved = sum(min(case["keep"], held) * max(0, held - case["keep"]) / max(1, held) for held in lens)
        return {"bytes": 8 * sum(lens) + moved * (4 * row + 16), "flops": 4.0 * sum(lens)}
    total = sum(new)
    if op == "append":
        return {"bytes": total * (4 * row + 12), "flops": total * 4.0}
    # query i of m sees all rows but the m - 1 - i last ones
    pairs = h * sum(m * held - m * (m - 1) / 2 for held, m in zip(lens, new) if held)
    rows = sum(held for held, m in zip(lens, new) if m)
    if op == "weights":
        return {"bytes": rows * row + 4 * sum(lens) + total * h * (d * e + 4), "flops": 2.0 * pairs * d}
    return {"bytes": 2 * rows * row + total * h * (2 * d * e + 4), "flops": 4.0 * pairs * d}


def exact(case, seed):
    global own
    kept, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = kept
    op = case["op"]
    if op in ("append", "evict"):
        return None                     # rows are copied, not computed
    if op == "logprobs":
        x = st["logits"].double()
        lp = torch.log_softmax(x, 1)
        out = {"logprob": lp[torch.arange(case["n"], device="cuda"), st["targets"].long()], "rank": None, "entropy": torch.special.entr(lp.exp()).sum(1)}
        if case["top"]:
            out["top_logprob"] = torch.full((case["n"], case["top"]), float("-inf"), dtype=torch.float64, device="cuda")
            best = torch.topk(lp, min(case["top"], case["vocab"]), 1).values
            out["top_logprob"][:, : best.shape[1]] = best
            out["top_token"] = None
        return out
    n, h, hkv, d, page = case["n_seq"], case["heads"], case["kv_heads"], case["dim"], case["page"]
    starts = list(range(n + 1)) if st["row_start"] is None else st["row_start"].tolist()
    out = torch.zeros(st["q"].shape[0], h, d, dtype=torch.float64, device="cuda")
    lses = torch.full((st["q"].shape[0], h), float("-inf"), dtype=torch.float64, device="cuda")
    weight = torch.zeros(st["weight"].shape, dtype=torch.float64, device="cuda")
    for b, held in enumerate(st["len"].tolist()):
        m = starts[b + 1] - starts[b]
        if held == 0 or (m == 0 and op == "attention"):
            continue
        pages = st["table"][b, : -(-held // page)].long()
        rows = {name: st[name][pages].flatten(0, 1)[:held].double() for name in ("k", "v")}
        gathered = torch.zeros(held, dtype=torch.float64, device="cuda")
        for head in range(h if m else 0):
            for first in range(0, m, 1024):
                part = slice(starts[b] + first, starts[b] + min(m, first + 1024))
                a = st["q"][part, head].double() @ rows["k"][:, head // (h // hkv)].T * d ** -0.5
                i = torch.arange(first, min(m, first + 1024), device="cuda")[:, None]
                a.masked_fill_(torch.arange(held, device="cuda")[None, :] > held - m + i, float("-inf"))
                if op == "weights":
                    gathered += torch.exp(a - st["lse"][part, head].double()[:, None]).sum(0)
                    continue
                lses[part, head] = torch.logsumexp(a, 1)
                out[part, head] = torch.softmax(a, 1) @ rows["v"][:, head // (h // hkv)]
        flat = torch.zeros(pages.numel() * page, dtype=torch.float64, device="cuda")
        flat[:held] = gathered / h
        weight[pages] = flat.view(-1, page)
    return weight if op == "weights" else {"out": out.reshape(-1, h * d), "lse": lses}
