"""Work of the block-cache operators: a paged key/value cache whose blocks are routed to like inverted lists.

A serving step takes requests with `cached` tokens in the cache and `fresh` new ones:

  tables     block tables, token positions and cache slots from the request lengths
  append     norm of queries and keys for each head, position rotation, and the write into the cache
  summarize  one 8-bit summary per block and kv head: the mean key, with a scale
  select     for each new token and kv head the blocks with the best summary score
  attend     attention of each new token over the blocks selected for it

Each case is one call of one of them.  With `own` false the operators run in their plain form, with `own`
true they are the framework's calls.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_MOST_GATHERED = 4096 * 4 * 16 * 64 * 128  # the largest listed attention, in gathered key elements


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one step of a small serving batch, one new token per request: only latency counts
        {"name": "tables_decode_32", "op": "tables", "requests": 32, "context": 32768, "prompts": 0, "chunk": 1, "page": 64},
        # a large mixed batch: one request in eight brings a prompt chunk, small pages, a 33 MB table
        {"name": "tables_mixed_2048", "op": "tables", "requests": 2048, "context": 65536, "prompts": 8, "chunk": 512, "page": 16},
        # a decode step with an odd batch, 7 query heads to a kv head, d = 96, two thirds of it rotated in pairs
        {"name": "append_decode_37_fp16", "op": "append", "tokens": 37, "kv_heads": 4, "group": 7, "dim": 96, "rotated": 64, "pairs": True, "page": 32, "type": "fp16"},
        # a long prompt chunk: bound by memory
        {"name": "append_prompt_16384", "op": "append", "tokens": 16384, "kv_heads": 8, "group": 4, "dim": 128, "rotated": 128, "pairs": False, "page": 64, "type": "bf16"},
        # after a decode step: the block that each request is filling
        {"name": "summarize_decode_64", "op": "summarize", "pages": 64, "filling": 64, "kv_heads": 8, "dim": 128, "page": 64, "type": "bf16"},
        # after prompts of half a million tokens, or when an index is rebuilt
        {"name": "summarize_prompt_8192", "op": "summarize", "pages": 8192, "filling": 16, "kv_heads": 8, "dim": 128, "page": 64, "type": "bf16"},
        # one user with a long context: latency
        {"name": "select_decode_1", "op": "select", "requests": 1, "context": 131072, "fresh": 1, "kv_heads": 8, "group": 4, "dim": 128, "page": 64, "take": 32, "type": "bf16"},
        # a decode batch over ragged contexts of up to 262,144 tokens: bound by the summaries' bytes
        {"name": "select_decode_32", "op": "select", "requests": 32, "context": 262144, "fresh": 1, "kv_heads": 8, "group": 4, "dim": 128, "page": 64, "take": 64, "type": "bf16"},
        # prompt chunks of two requests, every token with a selection of its own
        {"name": "select_prompt_4096_fp16", "op": "select", "requests": 2, "context": 32768, "fresh": 2048, "kv_heads": 4, "group": 8, "dim": 128, "page": 64, "take": 16, "type": "fp16"},
        # one user, odd head counts and a head width that is no power of two
        {"name": "attend_decode_1_fp16", "op": "attend", "requests": 1, "context": 131072, "fresh": 1, "kv_heads": 4, "group": 7, "dim": 96, "page": 64, "take": 32, "type": "fp16"},
        # a decode batch over ragged contexts: bound by the selected blocks' bytes
        {"name": "attend_decode_64", "op": "attend", "requests": 64, "context": 65536, "fresh": 1, "kv_heads": 8, "group": 4, "dim": 128, "page": 64, "take": 32, "type": "bf16"},
        # prompt chunks of two requests: bound by the products
        {"name": "attend_prompt_4096", "op": "attend", "requests": 2, "context": 32768, "fresh": 2048, "kv_heads": 4, "group": 8, "dim": 128, "page": 64, "take": 16, "type": "bf16"},
    ]


def _between(rng, low, high):
    """A whole number, spread over its logarithm."""
    return min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))


def draw(rng):
    op = rng.choice(["tables", "append", "summarize", "select", "attend", "attend"])
    page = rng.choice([16, 32, 64, 64, 128])
    if op == "tables":
        return {"op": op, "requests": _between(rng, 1, 2048), "context": _between(rng, 64, 65536), "prompts": rng.choice([0, 1, 3, 8]),
                "chunk": _between(rng, 1, 256), "page": page}
    dim = rng.choice([64, 80, 96, 128, 128, 256])
    kind = rng.choice(["bf16", "fp16"])
    heads = rng.choice([1, 2, 4, 8])
    if op == "append":
        group = rng.choice([1, 2, 3, 4, 7, 8, 16])
        most = 16384 * 48 * 128 // ((group + 2) * heads * dim)
        return {"op": op, "tokens": _between(rng, 1, min(16384, most)), "kv_heads": heads, "group": group, "dim": dim,
                "rotated": rng.choice([dim, dim // 32 * 16, 32]), "pairs": rng.random() < 0.3, "page": page, "type": kind}
    if op == "summarize":
        pages = _between(rng, 1, min(8192, 8192 * 64 * 8 * 128 // (page * heads * dim)))
        return {"op": op, "pages": pages, "filling": rng.randint(0, min(pages, 64)), "kv_heads": heads, "dim": dim, "page": page, "type": kind}
    group = rng.choice([1, 2, 4, 5, 7, 8, 16])
    take = rng.choice([4, 8, 16, 17, 32, 64])
    if rng.random() < 0.55:  # decode, some of it with a few drafted tokens
        requests, fresh = _between(rng, 1, 64), rng.choice([1, 1, 1, 2, 5])
    else:
        requests, fresh = rng.choice([1, 1, 2, 3, 5]), _between(rng, 16, 1024)
    context = _between(rng, 256, 131072)
    if op == "select":
        most = min(32 * 262144 // requests, 4 * 4096 * 2048 // (requests * fresh * heads) * page)
    else:
        most = 64 * 49152 * 8 * 128 // (requests * heads * dim)
        fresh = max(1, min(fresh, _MOST_GATHERED // (requests * heads * take * page * dim)))
    context = max(fresh, page, min(context, most))
    if op == "select":  # where all blocks are taken there is nothing to choose
        context = max(context, 2 * take * page)
    return {"op": op, "requests": requests, "context": context, "fresh": fresh, "kv_heads": heads, "group": group, "dim": dim, "page": page,
            "take": take, "type": kind}


def _lengths(case):
    """(tokens in the cache before the step, new tokens) of each request: ragged, by the case alone."""
    n = case["requests"]
    share = [1.0 if i == 0 else 0.25 + 0.75 * ((i * 0.6180339887) % 1.0) for i in range(n)]
    total = [max(1, int(case["context"] * s)) for s in share]
    if case["op"] == "tables":
        fresh = [(1 + (i * 7919) % case["chunk"]) if case["prompts"] and i % case["prompts"] == 0 else (0 if i % 17 == 16 else 1) for i in range(n)]
    else:
        fresh = [min(case["fresh"], t) for t in total]
    return [max(0, t - f) for t, f in zip(total, fresh)], fresh


def _up(a, b):
    return -(-a // b)


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _dev(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def prepare(case, seed):
    return {"tables": _prepare_tables, "append": _prepare_append, "summarize": _prepare_summarize, "select": _prepare_select,
            "attend": _prepare_attend}[case["op"]](case, _generator(seed))


def _prepare_tables(case, g):
    cached, fresh = _lengths(case)
    page = case["page"]
    old = [_up(c, page) for c in cached]
    most = max(_up(c + f, page) for c, f in zip(cached, fresh))
    columns = _up(most, 64) * 64
    held = sum(old)
    need = sum(_up(c + f, page) for c, f in zip(cached, fresh)) - held
    pool = torch.randperm(held + need + 64, device="cuda", generator=g).to(torch.int32)
    old_t = _dev(old, torch.int64)
    col = torch.arange(columns, device="cuda")
    place = (torch.cumsum(old_t, 0) - old_t)[:, None] + col[None]
    table = torch.where(col[None] < old_t[:, None], pool[place.clamp(max=held + need + 63)], -1).to(torch.int32).contiguous()
    tokens = _up(max(1, sum(fresh)), 64) * 64  # padded to a captured batch size
    return {"op": "tables", "page": page, "cached": _dev(cached), "fresh": _dev(fresh), "free": pool[held:].contiguous(), "table": table,
            "tokens": tokens, "touched": tokens // page + 2 * len(fresh)}


def _prepare_append(case, g):
    t, h, d, kind = case["tokens"], case["kv_heads"], case["dim"], _TYPES[case["type"]]
    hq, page = h * case["group"], case["page"]
    qkv = (torch.randn(t, (hq + 2 * h) * d, device="cuda", generator=g) * 1.5).to(kind)  # the projection's output
    pages = _up(t, page) + 2
    place = torch.randperm(pages * page, device="cuda", generator=g)[:t]
    limit = 8192
    angle = torch.arange(limit, device="cuda", dtype=torch.float64)[:, None] * torch.exp(
        torch.arange(0, case["rotated"], 2, device="cuda", dtype=torch.float64) * (-math.log(10000.0) / case["rotated"]))[None]
    weight = lambda: (1 + 0.1 * torch.randn(d, device="cuda", generator=g))  # noqa: E731
    return {"op": "append", "q": qkv[:, : hq * d].view(t, hq, d), "k": qkv[:, hq * d: (hq + h) * d].view(t, h, d), "v": qkv[:, (hq + h) * d:].view(t, h, d),
            "q_weight": weight(), "k_weight": weight(), "rotary": torch.cat([angle.cos(), angle.sin()], 1).float().contiguous(), "pairs": case["pairs"],
            "pos": torch.randint(0, limit, (t,), device="cuda", generator=g).to(torch.int32), "slot": place.to(torch.int64),
            "k_cache": torch.zeros(pages, h, page, d, device="cuda", dtype=kind), "v_cache": torch.zeros(pages, h, page, d, device="cuda", dtype=kind)}


def _keys(pages, h, page, d, kind, g):
    """Keys of a cache: tokens of a block lie around a centre of its own."""
    centre = torch.randn(pages, h, 1, d, device="cuda", generator=g, dtype=torch.float32)
    return torch.randn(pages, h, page, d, device="cuda", generator=g, dtype=kind).mul_(0.8).add_((0.6 * centre).to(kind))


def _prepare_summarize(case, g):
    n, h, d, page = case["pages"], case["kv_heads"], case["dim"], case["page"]
    keys = _keys(n, h, page, d, _TYPES[case["type"]], g)
    fill = torch.full((n,), page, device="cuda", dtype=torch.int32)
    fill[: case["filling"]] = torch.randint(1, page + 1, (case["filling"],), device="cuda", generator=g).to(torch.int32)
    return {"op": "summarize", "k_cache": keys, "pages": torch.randperm(n, device="cuda", generator=g).to(torch.int32), "fill": fill,
            "codes": torch.zeros(n, h, d, device="cuda", dtype=torch.int8), "scales": torch.zeros(n, h, device="cuda")}


def _prepare_step(case, g):
    """What select and attend have in hand: tables, tokens, queries."""
    cached, fresh = _lengths(case)
    page, h, d = case["page"], case["kv_heads"], case["dim"]
    blocks = [_up(c + f, page) for c, f in zip(cached, fresh)]
    columns, total = _up(max(blocks), 8) * 8, sum(blocks)
    held = _dev(blocks, torch.int64)
    pool = torch.randperm(total, device="cuda", generator=g).to(torch.int32)
    col = torch.arange(columns, device="cuda")
    place = (torch.cumsum(held, 0) - held)[:, None] + col[None]
    table = torch.where(col[None] < held[:, None], pool[place.clamp(max=total - 1)], -1).to(torch.int32).contiguous()
    tokens = sum(fresh)
    req = torch.repeat_interleave(torch.arange(len(fresh), device="cuda"), _dev(fresh, torch.int64), output_size=tokens)
    first = _dev(np.concatenate([[0], np.cumsum(fresh)[:-1]]).tolist(), torch.int64)
    pos = _dev(cached, torch.int64)[req] + torch.arange(tokens, device="cuda") - first[req]
    # neighbouring tokens ask for much the same: a direction shared by 64 of them and by a kv head's group, and noise of their own
    stretch = torch.arange(tokens, device="cuda") // 64 + req * 3
    shared = torch.randn(int(tokens // 64 + 3 * len(fresh) + 1), h, 1, d, device="cuda", generator=g)
    q = 0.95 * shared[stretch] + 0.3 * torch.randn(tokens, h, case["group"], d, device="cuda", generator=g)
    return {"page": page, "take": case["take"], "table": table, "req": req.to(torch.int32), "pos": pos.to(torch.int32),
            "q": (1.5 * q).reshape(tokens, h * case["group"], d).to(_TYPES[case["type"]])}, total


def _prepare_select(case, g):
    s, total = _prepare_step(case, g)
    h, d, page = case["kv_heads"], case["dim"], case["page"]
    mean = 0.6 * torch.randn(total, h, d, device="cuda", generator=g) + (0.8 / math.sqrt(page)) * torch.randn(total, h, d, device="cuda", generator=g)
    codes, scales = _coded(mean)
    return {"op": "select", **s, "codes": codes, "scales": scales}


def _prepare_attend(case, g):
    s, total = _prepare_step(case, g)
    h, d, page, kind = case["kv_heads"], case["dim"], case["page"], _TYPES[case["type"]]
    keys = _keys(total, h, page, d, kind, g)
    values = torch.randn(total, h, page, d, device="cuda", generator=g, dtype=kind)
    codes, scales = _coded(keys.mean(2, dtype=torch.float32))
    chosen = _select({**s, "codes": codes, "scales": scales})
    return {"op": "attend", **s, "k_cache": keys, "v_cache": values, "selected": chosen, "scale": 1.0 / math.sqrt(d)}


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _run_own(s)
    return {"tables": _tables, "append": _append, "summarize": _summarize, "select": _select, "attend": _attend}[s["op"]](s)


def _run_own(s):
    from paper_2608_08751_b200 import binding as B
    if s["op"] == "tables":
        p = B.ivf_kv_tables(s["cached"], s["fresh"], s["free"], s["table"], s["page"], s["tokens"])
        return [s["table"], p.kv_lens, p.token_start, p.token_req, p.token_pos, p.token_slot, p.touched_page, p.touched_fill, p.used]
    if s["op"] == "append":
        q = B.ivf_kv_append(s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["pos"], s["slot"], rotary=s["rotary"], interleaved=s["pairs"],
                            q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6)
        return [q, s["k_cache"], s["v_cache"]]
    if s["op"] == "summarize":
        B.ivf_kv_summarize(s["k_cache"], s["pages"], s["fill"], s["codes"], s["scales"])
        return [s["codes"] * s["scales"][..., None]]
    if s["op"] == "select":
        return B.ivf_kv_select(s["q"], s["codes"], s["scales"], s["table"], s["req"], s["pos"], s["page"], s["take"], n_first=1, n_last=2)
    return list(B.ivf_kv_attend(s["q"], s["k_cache"], s["v_cache"], s["table"], s["req"], s["pos"], s["selected"], s["scale"], want_lse=True))


# ------------------------------------------------------------------------------------------------ plain forms

def _tables(s):
    page, table = s["page"], s["table"]
    cached, fresh = s["cached"].long(), s["fresh"].long()
    total = cached + fresh
    old, now = (cached + page - 1) // page, (total + page - 1) // page
    need = now - old
    first = torch.cumsum(need, 0) - need
    col = torch.arange(table.shape[1], device=table.device)[None]
    new = s["free"][(first[:, None] + col - old[:, None]).clamp(0, s["free"].numel() - 1)]
    table.copy_(torch.where(col < old[:, None], table, torch.where(col < now[:, None], new, -1)))
    ends = torch.cumsum(fresh, 0)
    start = torch.cat([torch.zeros_like(ends[:1]), ends])
    t = torch.arange(s["tokens"], device=table.device)
    live = t < start[-1]
    req = torch.searchsorted(ends, t, right=True).clamp(max=fresh.numel() - 1)
    pos = cached[req] + t - start[req]
    block = torch.where(live, pos // page, 0)
    slot = table[req, block].long() * page + pos % page
    changed = torch.where(fresh > 0, now - cached // page, 0)
    until = torch.cumsum(changed, 0)
    w = torch.arange(s["touched"], device=table.device)
    there = w < until[-1]
    r = torch.searchsorted(until, w, right=True).clamp(max=fresh.numel() - 1)
    b = torch.where(there, cached[r] // page + w - (until - changed)[r], 0)
    fill = (total[r] - b * page).clamp(max=page)
    i32 = torch.int32
    return [table, total.to(i32), start.to(i32), torch.where(live, req, -1).to(i32), torch.where(live, pos, -1).to(i32), torch.where(live, slot, -1),
            torch.where(there, table[r, b], -1).to(i32), torch.where(there, fill, 0).to(i32), need.sum().to(i32).reshape(1)]


def _turned(x, weight, s):
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight
    cs = s["rotary"][s["pos"].long()][:, None]
    half = cs.shape[-1] // 2
    c, n = cs[..., :half], cs[..., half:]
    rest = x[..., 2 * half:]
    if s["pairs"]:
        a, b = x[..., 0: 2 * half: 2], x[..., 1: 2 * half: 2]
        return torch.cat([torch.stack([a * c - b * n, a * n + b * c], -1).flatten(-2), rest], -1)
    a, b = x[..., :half], x[..., half: 2 * half]
    return torch.cat([a * c - b * n, a * n + b * c, rest], -1)


def _append(s):
    page = s["k_cache"].shape[2]
    at, off = s["slot"] // page, s["slot"] % page
    s["k_cache"][at, :, off] = _turned(s["k"], s["k_weight"], s).to(s["k"].dtype)
    s["v_cache"][at, :, off] = s["v"]
    return [_turned(s["q"], s["q_weight"], s).to(s["q"].dtype), s["k_cache"], s["v_cache"]]


def _halved(x):
    """The sum over the first axis (a power of two long), the second half onto the first until one is left: the
    order of the additions is part of the definition, so that the codes are the same whole numbers everywhere."""
    n = x.shape[0] // 2
    return _halved(x[:n] + x[n:]) if n else x[0]


def _summed(x):
    """_halved() of any length, filled up with zeros."""
    n = 1 << (x.shape[0] - 1).bit_length()
    return _halved(x if n == x.shape[0] else torch.cat([x, x.new_zeros(n - x.shape[0], *x.shape[1:])]))


def _coded(x):
    """Rows of 32-bit numbers as whole numbers within +-127 and a scale."""
    scale = x.abs().amax(-1) * (1.0 / 127)  # one rounded factor
    scale = torch.where(scale >= 2.0 ** -126, scale, 0)
    code = torch.round(x / torch.where(scale > 0, scale, 1)[..., None]).clamp(-127, 127)
    return torch.where(scale[..., None] > 0, code, 0).to(torch.int8), scale


def _summarize(s):
    pages, fill = s["pages"].long(), s["fill"]
    page = s["k_cache"].shape[2]
    rows = s["k_cache"].movedim(2, 0)[:, pages].float()
    live = torch.arange(page, device=rows.device)[:, None] < fill[None]
    mean = _summed(torch.where(live[..., None, None], rows, 0)) / fill.float()[:, None, None]
    codes, scales = _coded(mean)
    s["codes"][pages], s["scales"][pages] = codes, scales
    return [s["codes"] * s["scales"][..., None]]


def _select(s):
    q, table, page, take = s["q"], s["table"], s["page"], s["take"]
    heads = s["codes"].shape[1]
    t = q.shape[0]
    query, _ = _coded(_summed(q.float().view(t, heads, -1, q.shape[2]).movedim(2, 0)))
    dots = torch.matmul(query.float().movedim(1, 0), s["codes"].float().movedim(1, 0).transpose(1, 2))  # whole numbers below 2^24: exact
    scores = (dots * s["scales"].t()[:, None]).movedim(0, 1)
    pages = table[s["req"].long()].long()
    scores = torch.gather(scores, 2, pages.clamp(min=0)[:, None].expand(-1, heads, -1))
    col, last = torch.arange(table.shape[1], device=q.device), (s["pos"] // page)[:, None, None]
    scores = torch.where((col < 1) | (col > last - 2), math.inf, scores)
    scores = torch.where((col <= last) & (pages >= 0)[:, None], scores, -math.inf)
    best = torch.sort(scores, dim=2, descending=True, stable=True)
    none = table.shape[1]
    ids = torch.where(best.values > -math.inf, best.indices, none)[..., :take]
    ids = torch.nn.functional.pad(ids, (0, take - ids.shape[2]), value=none)
    ids = torch.sort(ids, dim=2).values
    return torch.where(ids < none, ids, -1).to(torch.int32)


def _attend(s):
    q, chosen = s["q"], s["selected"].long()
    t, heads, take = chosen.shape
    page, d = s["k_cache"].shape[2:]
    at = torch.gather(s["table"][s["req"].long()].long(), 1, chosen.clamp(min=0).view(t, -1)).view(t, heads, take)
    place = chosen[..., None] * page + torch.arange(page, device=q.device)
    seen = ((chosen >= 0)[..., None] & (place <= s["pos"][:, None, None, None])).view(t, heads, 1, take * page)
    h = torch.arange(heads, device=q.device)[None, :, None]
    keys = s["k_cache"][at, h].view(t, heads, take * page, d).float()
    score = torch.matmul(q.float().view(t, heads, -1, d), keys.transpose(2, 3)) * s["scale"]
    del keys
    score = torch.where(seen, score, -math.inf)
    top = score.amax(3, keepdim=True).clamp(min=-3e38)
    p = torch.exp(score - top)
    total = p.sum(3, keepdim=True)
    values = s["v_cache"][at, h].view(t, heads, take * page, d).float()
    out = torch.matmul(p, values) / torch.where(total > 0, total, 1)
    return [out.reshape(q.shape).to(q.dtype), (torch.log(total) + top).reshape(q.shape[:2])]


# ------------------------------------------------------------------------------------------------ work

def work(case):
    op, page = case["op"], case["page"]
    if op == "tables":
        cached, fresh = _lengths(case)
        columns = _up(max(_up(c + f, page) for c, f in zip(cached, fresh)), 64) * 64
        held = sum(_up(c, page) for c in cached)
        tokens = _up(max(1, sum(fresh)), 64) * 64
        n = len(fresh)
        # lengths in, table entries past the held ones out, tokens (request, position, slot), touched blocks
        return {"bytes": 8 * n + 4 * (n * columns - held) + 16 * tokens + 8 * (tokens // page + 2 * n) + 8 * n, "flops": 0}
    h, d = case["kv_heads"], case["dim"]
    if op == "append":
        t, hq = case["tokens"], h * case["group"]
        return {"bytes": 4 * t * (hq + 2 * h) * d + t * (12 + 4 * case["rotated"]), "flops": t * (hq + h) * d * 8}
    if op == "summarize":
        n, part = case["pages"], case["filling"]
        read = (n - part) * page + part * (page + 1) // 2
        return {"bytes": read * h * d * 2 + n * h * (d + 4), "flops": read * h * d}
    cached, fresh = _lengths(case)
    tokens, hq, take = sum(fresh), h * case["group"], case["take"]
    if op == "select":
        blocks = [_up(c + f, page) for c, f in zip(cached, fresh)]
        return {"bytes": tokens * hq * d * 2 + sum(blocks) * (h * (d + 4) + 4) + tokens * h * take * 4 + tokens * 8,
                "flops": 2 * h * d * sum(f * b for f, b in zip(fresh, blocks))}
    seen = [min(c + f, take * page) for c, f in zip(cached, fresh)]
    read = sum(min(f * s, c + f) for c, f, s in zip(cached, fresh, seen))
    return {"bytes": read * h * d * 4 + tokens * hq * (d * 4 + 4) + tokens * h * take * 4, "flops": 4 * hq * d * sum(f * s for f, s in zip(fresh, seen))}


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    return {"tables": _exact_tables, "append": _exact_append, "summarize": _exact_summarize, "select": _exact_select,
            "attend": _exact_attend}[case["op"]](prepare(case, seed))


def _exact_tables(s):
    page = s["page"]
    cached, fresh, free, table = (s[k].cpu().numpy().astype(np.int64) for k in ("cached", "fresh", "free", "table"))
    req, pos, slot = (np.full(s["tokens"], -1, np.int64) for _ in range(3))
    touched, fill = np.full(s["touched"], -1, np.int64), np.zeros(s["touched"], np.int64)
    used = n = m = 0
    start = [0]
    for b, (c, f) in enumerate(zip(cached.tolist(), fresh.tolist())):
        old, now = _up(c, page), _up(c + f, page)
        table[b, old:now] = free[used: used + now - old]
        table[b, now:] = -1
        used += now - old
        p = np.arange(c, c + f)
        req[n: n + f], pos[n: n + f], slot[n: n + f] = b, p, table[b, p // page] * page + p % page
        n += f
        start.append(n)
        if f:
            j = np.arange(c // page, now)
            touched[m: m + len(j)], fill[m: m + len(j)] = table[b, j], np.minimum(page, c + f - j * page)
            m += len(j)
    i = lambda a: np.asarray(a, np.int32)  # noqa: E731
    return [i(table), i(cached + fresh), i(start), i(req), i(pos), slot, i(touched), i(fill), i([used])]


def _exact_append(s):
    def turn(x, weight):
        x = x.double()
        y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.double()
        cs = s["rotary"].double()[s["pos"].long()]
        half = cs.shape[1] // 2
        z = torch.complex(cs[:, :half], cs[:, half:])[:, None]
        first = torch.arange(half, device=x.device) * (2 if s["pairs"] else 1)
        second = first + (1 if s["pairs"] else half)
        w = torch.complex(y[..., first], y[..., second]) * z
        y[..., first], y[..., second] = w.real, w.imag
        return y
    page = s["k_cache"].shape[2]
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    k_cache.movedim(1, 2)[s["slot"] // page, s["slot"] % page] = turn(s["k"], s["k_weight"])
    v_cache.movedim(1, 2)[s["slot"] // page, s["slot"] % page] = s["v"].double()
    return [turn(s["q"], s["q_weight"]), k_cache, v_cache]


def _exact_summarize(s):
    n, h, page, d = s["k_cache"].shape
    out = torch.zeros(n, h, d, device="cuda", dtype=torch.float64)
    for i in range(0, n, 512):
        at, fill = s["pages"][i: i + 512].long(), s["fill"][i: i + 512]
        live = (torch.arange(page, device="cuda") < fill[:, None]).double()
        mean = torch.einsum("nhpd,np->nhd", s["k_cache"][at].double(), live) / fill.double()[:, None, None]
        unit = mean.abs().amax(2, keepdim=True) / 127
        out[at] = torch.where(unit > 0, torch.round(mean / unit) * unit, 0)
    return [out]


def _exact_select(s):
    q, codes, scales = s["q"].float(), s["codes"].long(), s["scales"]
    t, heads, d = q.shape[0], codes.shape[1], codes.shape[2]
    query, _ = _coded(_summed(q.view(t, heads, -1, d).movedim(2, 0)))  # the query's codes are part of the definition
    out = torch.full((t, heads, s["take"]), -1, dtype=torch.int32)
    if t * heads > 512:
        return None
    for i in range(t):
        r, last = int(s["req"][i]), int(s["pos"][i]) // s["page"]
        pages = s["table"][r, : last + 1].long()
        dots = (query[i].double()[None] * codes[pages].double()).sum(-1)
        score = (dots * scales[pages].double()).float().cpu().numpy()  # one rounding to 32 bits
        score[:1] = math.inf
        score[max(0, last - 1):] = math.inf
        for h in range(heads):
            best = np.sort(np.argsort(-score[:, h], kind="stable")[: s["take"]])
            out[i, h, : len(best)] = torch.from_numpy(best)
    return out


def _exact_attend(s):
    q, chosen = s["q"].double(), s["selected"].long()
    t, heads, take = chosen.shape
    page, d = s["k_cache"].shape[2:]
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda", dtype=torch.float64)
    step = max(1, 100_000_000 // (heads * take * page * d))
    h = torch.arange(heads, device="cuda")[None, :, None]
    for i in range(0, t, step):
        c = chosen[i: i + step]
        n = c.shape[0]
        at = s["table"].long()[s["req"][i: i + n].long()[:, None, None], c.clamp(min=0)]
        k = s["k_cache"][at, h].reshape(n, heads, take * page, d).double()
        v = s["v_cache"][at, h].reshape(n, heads, take * page, d).double()
        place = (c[..., None] * page + torch.arange(page, device="cuda")).reshape(n, heads, 1, -1)
        seen = (place <= s["pos"][i: i + n].long()[:, None, None, None]) & (c >= 0).repeat_interleave(page, 2)[:, :, None]
        z = (q[i: i + n].view(n, heads, -1, d) @ k.transpose(2, 3) * s["scale"]).masked_fill(~seen, -math.inf)
        out[i: i + n] = (torch.softmax(z, 3) @ v).reshape(n, -1, d)
        lse[i: i + n] = torch.logsumexp(z, 3).reshape(n, -1)
    return [out, lse]
