"""Work of the operators that keep a whole paged cache in use: attention of new tokens over all of it, and the life of its pages.

A server of a language model whose layers read the whole cache (or a window of it) has, beside the block tables:

  chunk    attention of each request's new tokens (a prompt's chunk, one token, a few drafted ones) over its pages: causal, with
           a window, a prefix that all its tokens see, scores capped by a tanh, a bias that falls with the distance
  fork     the tables of the next step from those of this one: rows that continue, branch, are cut back or end; full pages are
           shared, a partly filled one has one owner and copies; the pages that nobody holds
  compact  pages past the number of held ones move into holes below it; the tables that say so
  copy     the pages of a list onto the pages of another, in one layer's cache

Each case is one call of one of them.  With `own` false the operators run in their plain form, with `own`
true they are the framework's calls.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_MOST_PRODUCTS = 4096 * 32 * 30000 * 128  # below the largest listed chunk: tokens x query heads x keys x head width
_MOST_CACHE = 131072 * 8 * 128            # its longest cache, in key elements


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one user with a long context, one token at a time: bound by the cache's bytes
        {"name": "chunk_decode_1", "op": "chunk", "requests": 1, "context": 131072, "fresh": 1, "kv_heads": 8, "group": 4, "dim": 128, "page": 64,
         "cap": 0.0, "bias": False, "window": 0, "prefix": 0, "type": "bf16"},
        # a small decode batch of capped scores over a window: latency; odd heads, a head width that is no power of two
        {"name": "chunk_decode_37_window_fp16", "op": "chunk", "requests": 37, "context": 20000, "fresh": 1, "kv_heads": 4, "group": 7, "dim": 96, "page": 32,
         "cap": 30.0, "bias": False, "window": 1000, "prefix": 0, "type": "fp16"},
        # drafted tokens of a batch, heads without groups, a bias by distance, small pages, ragged contexts
        {"name": "chunk_draft_24_bias", "op": "chunk", "requests": 24, "context": 16384, "fresh": 5, "kv_heads": 16, "group": 1, "dim": 64, "page": 16,
         "cap": 0.0, "bias": True, "window": 0, "prefix": 0, "type": "bf16"},
        # prompt chunks of two requests far into their contexts: bound by the products
        {"name": "chunk_prompt_4096", "op": "chunk", "requests": 2, "context": 32768, "fresh": 2048, "kv_heads": 4, "group": 8, "dim": 128, "page": 64,
         "cap": 0.0, "bias": False, "window": 0, "prefix": 0, "type": "bf16"},
        # a whole prompt at once, its first part (an image, a document) seen by all of it
        {"name": "chunk_prompt_prefix_fp16", "op": "chunk", "requests": 1, "context": 8001, "fresh": 8001, "kv_heads": 8, "group": 4, "dim": 128, "page": 64,
         "cap": 0.0, "bias": False, "window": 0, "prefix": 1500, "type": "fp16"},
        # wide heads with capped scores and a window, ragged prompt chunks
        {"name": "chunk_prompt_cap_window", "op": "chunk", "requests": 3, "context": 16384, "fresh": 1500, "kv_heads": 4, "group": 2, "dim": 256, "page": 128,
         "cap": 50.0, "bias": False, "window": 4096, "prefix": 0, "type": "bf16"},
        # a step of a beam search: 8 requests of 4 beams, only latency counts
        {"name": "fork_beams_32", "op": "fork", "rows": 32, "beams": 4, "context": 8192, "cut": 0, "page": 64},
        # a large batch of small pages: requests that end, branch, and are cut back after a refused draft
        {"name": "fork_mixed_1024", "op": "fork", "rows": 1024, "beams": 2, "context": 32768, "cut": 8, "page": 16},
        # a small server that gives memory back
        {"name": "compact_64", "op": "compact", "rows": 64, "context": 4096, "holes": 3, "page": 64},
        # a cache of half a million pages after its batch has halved
        {"name": "compact_512", "op": "compact", "rows": 512, "context": 32768, "holes": 2, "page": 16},
        # the partly filled pages of forked beams
        {"name": "copy_beams_32_fp16", "op": "copy", "pages": 32, "partial": True, "kv_heads": 4, "dim": 96, "page": 32, "type": "fp16"},
        # the moves of a compaction in one layer: bound by memory
        {"name": "copy_moves_4096", "op": "copy", "pages": 4096, "partial": False, "kv_heads": 8, "dim": 128, "page": 64, "type": "bf16"},
    ]


def _between(rng, low, high):
    """A whole number, spread over its logarithm."""
    return min(high, int(math.exp(rng.uniform(math.log(low), math.log(high + 1)))))


def draw(rng):
    op = rng.choice(["chunk", "chunk", "chunk", "chunk", "fork", "compact", "copy"])
    page = rng.choice([16, 32, 64, 64, 128])
    if op in ("fork", "compact"):
        context = _between(rng, 64, 32768)
        rows = _between(rng, 1, max(1, min(1024, 1024 * 2048 * page // max(context, page))))
        if op == "fork":
            return {"op": op, "rows": rows, "beams": rng.choice([1, 2, 4, 5, 8]), "context": context, "cut": rng.choice([0, 0, 3, 8]), "page": page}
        return {"op": op, "rows": min(rows, 512), "context": context, "holes": rng.choice([2, 3, 5, 50]), "page": page}
    heads = rng.choice([1, 2, 4, 8])
    dim = rng.choice([64, 80, 96, 128, 128, 256])
    kind = rng.choice(["bf16", "fp16"])
    if op == "copy":
        pages = _between(rng, 1, min(4096, 4096 * 64 * 8 * 128 // (page * heads * dim)))
        return {"op": op, "pages": pages, "partial": rng.random() < 0.5, "kv_heads": heads, "dim": dim, "page": page, "type": kind}
    group = rng.choice([1, 2, 4, 5, 7, 8, 16])
    if rng.random() < 0.5:  # decode, some of it with a few drafted tokens
        requests, fresh = _between(rng, 1, 64), rng.choice([1, 1, 1, 2, 5])
        context = _between(rng, 64, 131072)
    else:
        requests, fresh = rng.choice([1, 1, 2, 3, 5]), _between(rng, 16, 4096)
        context = _between(rng, 64, 32768) if rng.random() < 0.6 else fresh  # far into a context, or a prompt from its start
    context = max(page, min(context, _MOST_CACHE // (requests * heads * dim)))
    fresh = min(fresh, context)
    while requests * fresh * heads * group * dim * context > _MOST_PRODUCTS:
        fresh = (fresh + 1) // 2
    return {"op": op, "requests": requests, "context": context, "fresh": fresh, "kv_heads": heads, "group": group, "dim": dim, "page": page,
            "cap": rng.choice([0.0, 0.0, 0.0, 20.0, 50.0]), "bias": rng.random() < 0.25, "window": rng.choice([0, 0, 0, _between(rng, 1, 8192)]),
            "prefix": rng.choice([0, 0, 0, _between(rng, 1, context)]), "type": kind}


def _up(a, b):
    return -(-a // b)


def _shares(n):
    return [1.0 if i == 0 else 0.25 + 0.75 * ((i * 0.6180339887) % 1.0) for i in range(n)]


def _lengths(case):
    """(tokens in the cache with the new ones, new tokens) of each request of a chunk: ragged, by the case alone."""
    total = [max(1, int(case["context"] * s)) for s in _shares(case["requests"])]
    fresh = [max(1, min(case["fresh"] - (i * 7919) % max(1, case["fresh"] // 3), t)) for i, t in enumerate(total)]
    return total, fresh


def _row_lengths(case):
    return [max(1, int(case["context"] * s)) for s in _shares(case["rows"])]


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _dev(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def prepare(case, seed):
    return {"chunk": _prepare_chunk, "fork": _prepare_fork, "compact": _prepare_compact, "copy": _prepare_copy}[case["op"]](case, _generator(seed))


def _tables(blocks, columns, pool):
    """Rows of `blocks` pages each, taken from the front of the pool."""
    held = _dev(blocks, torch.int64)
    col = torch.arange(columns, device="cuda")
    place = (torch.cumsum(held, 0) - held)[:, None] + col[None]
    return torch.where(col[None] < held[:, None], pool[place.clamp(max=pool.numel() - 1)], -1).to(torch.int32).contiguous()


def _prepare_chunk(case, g):
    total, fresh = _lengths(case)
    page, h, d, kind = case["page"], case["kv_heads"], case["dim"], _TYPES[case["type"]]
    heads = h * case["group"]
    blocks = [_up(t, page) for t in total]
    pages = sum(blocks)
    table = _tables(blocks, _up(max(blocks), 8) * 8, torch.randperm(pages, device="cuda", generator=g))
    start = [0]
    for f in fresh:
        start.append(start[-1] + f)
    # keys of a cache: tokens of a block lie around a centre of its own
    centre = torch.randn(pages, h, 1, d, device="cuda", generator=g, dtype=torch.float32)
    keys = torch.randn(pages, h, page, d, device="cuda", generator=g, dtype=kind).mul_(0.8).add_((0.6 * centre).to(kind))
    values = torch.randn(pages, h, page, d, device="cuda", generator=g, dtype=kind)
    q = (1.5 * torch.randn(start[-1], heads, d, device="cuda", generator=g)).to(kind)
    slopes = torch.exp2(-8.0 * torch.arange(1, heads + 1, device="cuda", dtype=torch.float32) / heads) if case["bias"] else None
    prefix = _dev([max(0, case["prefix"] - 37 * i) for i in range(len(total))]) if case["prefix"] else None
    return {"op": "chunk", "q": q, "k_cache": keys, "v_cache": values, "table": table, "start": _dev(start), "lens": _dev(total),
            "scale": 1.0 / math.sqrt(d), "cap": case["cap"], "slopes": slopes, "window": case["window"], "prefix": prefix,
            "lengths": list(zip(start, fresh, total)), "host_prefix": prefix.tolist() if prefix is not None else [0] * len(total)}


def _prepare_fork(case, g):
    page, rows = case["page"], case["rows"]
    lens = _row_lengths(case)
    blocks = [_up(t, page) for t in lens]
    pages = sum(blocks) + rows + 64
    table = _tables(blocks, _up(max(blocks), 8) * 8, torch.randperm(pages, device="cuda", generator=g))
    # beams of a request share their first half already, the full pages of it
    row = torch.arange(rows, device="cuda")
    first = row // case["beams"] * case["beams"]
    least = _dev(lens, torch.int64)
    shared = torch.minimum(least, least[first]) // 2 // page
    col = torch.arange(table.shape[1], device="cuda")[None]
    table = torch.where(col < shared[:, None], table[first], table).contiguous()
    parent = (first + torch.randint(0, case["beams"], (rows,), device="cuda", generator=g)).clamp(max=rows - 1)
    keep = least[parent]
    if case["cut"]:  # every so many rows: ends, or loses its last few tokens
        some = row % case["cut"]
        keep = torch.where(some == 1, (keep - 1 - row % 11).clamp(min=0), keep)
        parent = torch.where(some == 2, -1, parent)
    return {"op": "fork", "page": page, "pages": pages, "table": table, "lens": least.to(torch.int32), "parent": parent.to(torch.int32),
            "keep": torch.where(parent < 0, 0, keep).to(torch.int32)}


def _prepare_compact(case, g):
    page, rows = case["page"], case["rows"]
    lens = _row_lengths(case)
    blocks = [_up(t, page) for t in lens]
    pages = sum(blocks) + 64
    table = _tables(blocks, _up(max(blocks), 8) * 8, torch.randperm(pages, device="cuda", generator=g))
    ended = torch.arange(rows, device="cuda") % case["holes"] == case["holes"] - 1  # requests that have ended
    lens = torch.where(ended, 0, _dev(lens))
    return {"op": "compact", "page": page, "pages": pages, "table": table, "lens": lens.to(torch.int32).contiguous()}


def _prepare_copy(case, g):
    n, h, d, page, kind = case["pages"], case["kv_heads"], case["dim"], case["page"], _TYPES[case["type"]]
    total = 2 * n + 7
    place = torch.randperm(total, device="cuda", generator=g).to(torch.int32)
    fill = torch.randint(1, page + 1, (n,), device="cuda", generator=g).to(torch.int32) if case["partial"] else None
    return {"op": "copy", "k_cache": torch.randn(total, h, page, d, device="cuda", generator=g, dtype=kind),
            "v_cache": torch.randn(total, h, page, d, device="cuda", generator=g, dtype=kind), "from": place[:n].contiguous(),
            "to": place[n: 2 * n].contiguous(), "fill": fill}


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    if own:
        return _run_own(s)
    return {"chunk": _chunk, "fork": _fork, "compact": _compact, "copy": _copy}[s["op"]](s)


def _run_own(s):
    from paper_2608_08751_b200 import binding as B
    if s["op"] == "chunk":
        return list(B.ivf_kv_attend_chunk(s["q"], s["k_cache"], s["v_cache"], s["table"], s["start"], s["lens"], s["scale"], cap=s["cap"],
                                          slopes=s["slopes"], window=s["window"], prefix=s["prefix"], want_lse=True))
    if s["op"] == "fork":
        return list(B.ivf_kv_fork(s["table"], s["lens"], s["parent"], s["keep"], s["pages"], s["page"]))
    if s["op"] == "compact":
        return list(B.ivf_kv_compact(s["table"], s["lens"], s["pages"], s["page"], out=torch.empty_like(s["table"])))
    B.ivf_kv_copy(s["k_cache"], s["v_cache"], s["from"], s["to"], s["fill"])
    return [s["k_cache"], s["v_cache"]]


# ------------------------------------------------------------------------------------------------ plain forms

def _chunk(s):
    q, page = s["q"], s["k_cache"].shape[2]
    heads, d = s["k_cache"].shape[1], q.shape[2]
    group = q.shape[1] // heads
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], device=q.device)
    for b, (t0, fresh, total) in enumerate(s["lengths"]):
        at = s["table"][b, : _up(total, page)].long()
        pos = torch.arange(total - fresh, total, device=q.device)[:, None]
        key = torch.arange(total, device=q.device)[None]
        seen = (key <= pos) | (key < s["host_prefix"][b])
        if s["window"]:
            seen &= pos - key < s["window"]
        away = (pos - key).abs().float()
        for h in range(heads):
            k = s["k_cache"][at, h].reshape(-1, d)[:total].float()
            v = s["v_cache"][at, h].reshape(-1, d)[:total].float()
            for i in range(h * group, (h + 1) * group):
                score = torch.matmul(q[t0: t0 + fresh, i].float(), k.t()) * s["scale"]
                if s["cap"]:
                    score = s["cap"] * torch.tanh(score / s["cap"])
                if s["slopes"] is not None:
                    score = score - s["slopes"][i] * away
                score = torch.where(seen, score, -math.inf)
                top = score.amax(1, keepdim=True)
                p = torch.exp(score - top)
                sums = p.sum(1, keepdim=True)
                out[t0: t0 + fresh, i] = (torch.matmul(p, v) / sums).to(q.dtype)
                lse[t0: t0 + fresh, i] = (torch.log(sums) + top)[:, 0]
    return [out, lse]


def _numbered(free, n):
    """The whole numbers below n where `free` holds, ascending, -1 after the last."""
    place = torch.cumsum(free.long(), 0) - 1
    out = torch.full((n + 1,), -1, dtype=torch.int64, device=free.device)
    out[torch.where(free, place, n)] = torch.arange(free.numel(), device=free.device)
    out[n] = -1
    return out[:n]


def _fork(s):
    page, pages, table = s["page"], s["pages"], s["table"]
    n, columns = s["parent"].numel(), table.shape[1]
    live = s["parent"] >= 0
    parent = s["parent"].long().clamp(min=0)
    keep = torch.where(live, torch.minimum(s["keep"].long(), s["lens"].long()[parent]), 0)
    col = torch.arange(columns, device=table.device)[None]
    full, rest = keep // page, keep % page
    old = table[parent].long()
    held = torch.zeros(pages + 1, dtype=torch.bool, device=table.device)
    held[torch.where(col < full[:, None], old, pages).flatten()] = True
    has = rest > 0
    last = torch.where(has, torch.gather(old, 1, full.clamp(max=columns - 1)[:, None])[:, 0], pages)
    row = torch.arange(n, device=table.device)
    first = torch.full((pages + 1,), n, dtype=torch.int64, device=table.device).scatter_reduce(0, last, row, "amin")
    owner = has & ~held[last] & (first[last] == row)
    copied = has & ~owner
    held[last] = True
    free = _numbered(~held[:pages], pages)
    rank = torch.cumsum(copied.long(), 0) - 1
    to = torch.where(copied, free[rank.clamp(min=0)], -1)
    taken = copied.sum()
    new = torch.where(col < full[:, None], old, -1)
    tail = torch.where(owner, last, to)
    new = torch.where((col == full[:, None]) & has[:, None], tail[:, None], new)
    at = torch.arange(pages, device=table.device) + taken
    left = torch.where(at < pages, free[at.clamp(max=pages - 1)], -1)
    i32 = torch.int32
    return [new.to(i32), keep.to(i32), torch.where(copied, last, -1).to(i32), to.to(i32), torch.where(copied, rest, 0).to(i32), left.to(i32),
            ((~held[:pages]).sum() - taken).to(i32).reshape(1)]


def _compact(s):
    page, pages, table = s["page"], s["pages"], s["table"]
    blocks = (s["lens"].long() + page - 1) // page
    inside = torch.arange(table.shape[1], device=table.device)[None] < blocks[:, None]
    held = torch.zeros(pages + 1, dtype=torch.bool, device=table.device)
    held[torch.where(inside, table.long(), pages).flatten()] = True
    held = held[:pages]
    count = held.sum()
    number = torch.arange(pages, device=table.device)
    to = _numbered(~held & (number < count), pages)
    moving = (held & (number >= count)).flip(0)  # the highest first
    source = _numbered(moving, pages)
    source = torch.where(source >= 0, pages - 1 - source, -1)
    new = torch.cat([number, number[:1]])
    new[torch.where(source >= 0, source, pages)] = torch.where(source >= 0, to, -1)
    i32 = torch.int32
    out = torch.where(inside, new[table.long().clamp(min=0)], -1)
    return [out.to(i32), source.to(i32), to.to(i32), count.to(i32).reshape(1)]


def _copy(s):
    a, b = s["from"].long(), s["to"].long()
    for cache in (s["k_cache"], s["v_cache"]):
        if s["fill"] is None:
            cache[b] = cache[a]
        else:
            inside = torch.arange(cache.shape[2], device=cache.device)[None] < s["fill"][:, None]
            cache[b] = torch.where(inside[:, None, :, None], cache[a], cache[b])
    return [s["k_cache"], s["v_cache"]]


# ------------------------------------------------------------------------------------------------ work

def _seen(case):
    """(keys that some token of a request sees, pairs of a token and a key) of each request."""
    total, fresh = _lengths(case)
    out = []
    for b, (n, f) in enumerate(zip(total, fresh)):
        pos = np.arange(n - f, n)
        prefix = max(0, case["prefix"] - 37 * b) if case["prefix"] else 0
        low = np.maximum(0, pos - case["window"] + 1) if case["window"] else np.zeros(f, np.int64)
        high = np.maximum(pos + 1, min(prefix, n))
        out.append((int(high.max() - low.min()), int((high - low).sum())))
    return out


def work(case):
    op, page = case["op"], case["page"]
    if op == "chunk":
        total, fresh = _lengths(case)
        heads, d = case["kv_heads"] * case["group"], case["dim"]
        seen = _seen(case)
        keys, pairs = sum(k for k, _ in seen), sum(p for _, p in seen)
        return {"bytes": keys * case["kv_heads"] * d * 4 + sum(fresh) * heads * (d * 4 + 4) + 4 * sum(_up(k, page) for k, _ in seen), "flops": 4 * heads * d * pairs}
    if op == "copy":
        tokens = case["pages"] * (page + 1) // 2 if case["partial"] else case["pages"] * page
        return {"bytes": tokens * case["kv_heads"] * case["dim"] * 8, "flops": 0}
    lens = _row_lengths(case)
    blocks = [_up(t, page) for t in lens]
    columns = _up(max(blocks), 8) * 8
    if op == "fork":  # the held entries in, whole rows out; lengths, parents, copies; the list of free pages
        return {"bytes": 4 * sum(blocks) + 4 * case["rows"] * (columns + 7) + 4 * (sum(blocks) + case["rows"] + 64), "flops": 0}
    held = sum(b for i, b in enumerate(blocks) if i % case["holes"] != case["holes"] - 1)
    return {"bytes": 4 * held + 4 * case["rows"] * (columns + 1) + 8 * (sum(blocks) + 64), "flops": 0}


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    return {"chunk": _exact_chunk, "fork": _exact_fork, "compact": _exact_compact, "copy": _exact_copy}[case["op"]](prepare(case, seed))


def _exact_chunk(s):
    q = s["q"].double()
    pages, heads, page, d = s["k_cache"].shape
    n_heads = q.shape[1]
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, device="cuda", dtype=torch.float64)
    for b in range(s["lens"].numel()):
        t0, t1, n = int(s["start"][b]), int(s["start"][b + 1]), int(s["lens"][b])
        rows = s["table"][b, torch.arange(n, device="cuda") // page].long() * page + torch.arange(n, device="cuda") % page  # of each token
        for g in range(n_heads):
            h = g // (n_heads // heads)
            k = s["k_cache"][:, h].reshape(-1, d)[rows].double()
            v = s["v_cache"][:, h].reshape(-1, d)[rows].double()
            for i in range(t0, t1, 1024):
                j = min(t1, i + 1024)
                distance = torch.arange(n - t1 + i, n - t1 + j, device="cuda")[:, None] - torch.arange(n, device="cuda")
                hidden = distance < 0
                if s["prefix"] is not None:
                    hidden &= torch.arange(n, device="cuda") >= s["prefix"][b]
                if s["window"] > 0:
                    hidden |= distance >= s["window"]
                z = torch.einsum("td,kd->tk", q[i:j, g], k) * s["scale"]
                if s["cap"] > 0:
                    z = s["cap"] * torch.tanh(z / s["cap"])
                if s["slopes"] is not None:
                    z = z - s["slopes"][g].double() * distance.abs()
                z = z.masked_fill(hidden, -math.inf)
                out[i:j, g] = torch.softmax(z, 1) @ v
                lse[i:j, g] = torch.logsumexp(z, 1)
    return [out, lse]


def _exact_fork(s):
    page, pages = s["page"], s["pages"]
    table, lens, parent, keep = (s[k].cpu().numpy().astype(np.int64) for k in ("table", "lens", "parent", "keep"))
    n = len(parent)
    new = np.full((n, table.shape[1]), -1, np.int64)
    kept = np.array([min(k, lens[p]) if p >= 0 else 0 for p, k in zip(parent, keep)])
    shared = set()
    for i in range(n):
        full = kept[i] // page
        new[i, :full] = table[parent[i], :full]
        shared.update(new[i, :full].tolist())
    source, to, fill = np.full(n, -1), np.full(n, -1), np.zeros(n, np.int64)
    owned, waiting = set(), []
    for i in range(n):
        if kept[i] % page:
            p = table[parent[i], kept[i] // page]
            if p in shared or p in owned:
                waiting.append(i)
                source[i], fill[i] = p, kept[i] % page
            else:
                owned.add(p)
                new[i, kept[i] // page] = p
    free = sorted(set(range(pages)) - shared - owned)
    for i in waiting:
        to[i] = new[i, kept[i] // page] = free.pop(0) if len(waiting) < 64 else free[len(to[to >= 0])]
    if len(waiting) >= 64:
        free = free[len(waiting):]
    i32 = lambda a: np.asarray(a, np.int32)  # noqa: E731
    return [i32(new), i32(kept), i32(source), i32(to), i32(fill), i32(free + [-1] * (pages - len(free))), i32([len(free)])]


def _exact_compact(s):
    page, pages = s["page"], s["pages"]
    table, lens = s["table"].cpu().numpy().astype(np.int64), s["lens"].cpu().numpy()
    rows = [table[b, : _up(int(n), page)] for b, n in enumerate(lens)]
    held = np.unique(np.concatenate(rows))
    high = held[held >= len(held)][::-1]
    low = np.setdiff1d(np.arange(len(held)), held)
    where = np.arange(pages)
    where[high] = low
    out = np.full_like(table, -1)
    for b, r in enumerate(rows):
        out[b, : len(r)] = where[r]
    pad = np.full(pages - len(high), -1)
    i32 = lambda a: np.asarray(a, np.int32)  # noqa: E731
    return [i32(out), i32(np.concatenate([high, pad])), i32(np.concatenate([low, pad])), i32([len(held)])]


def _exact_copy(s):
    return None if s["k_cache"].shape[0] > 2000 else [_copied(s["k_cache"], s), _copied(s["v_cache"], s)]


def _copied(cache, s):
    new = cache.double()
    for i, (a, b) in enumerate(zip(s["from"].tolist(), s["to"].tolist())):
        n = cache.shape[2] if s["fill"] is None else int(s["fill"][i])
        new[b, :, :n] = cache[a, :, :n].double()
    return new
