"""Plain 64-bit forms of the operators on whole paged caches, written from their definitions in numpy; nothing is shared with the
library."""
import math

import numpy as np


def attend_chunk(q, k_cache, v_cache, table, start, lens, scale, cap=0.0, slopes=None, window=0, prefix=None):
    """(out, lse, attention-weighted mean of |v|, largest magnitude that meets in a logit): q [n, heads, d], caches [pages, kv_heads, page, d],
    float64.  A page outside the cache is missing."""
    n, heads, d = q.shape
    pages, kv, page = k_cache.shape[:3]
    out, size = np.zeros((n, heads, d)), np.zeros((n, heads, d))
    lse, unit = np.full((n, heads), -np.inf), np.zeros((n, heads))
    for b in range(len(lens)):
        given = int(start[b + 1]) - int(start[b])
        if given < 0 or int(lens[b]) < given:
            continue
        for t in range(int(start[b]), min(int(start[b + 1]), n)):
            pos = int(lens[b]) - given + t - int(start[b])
            keys = np.arange(int(lens[b]))
            seen = (keys <= pos) | (keys < (prefix[b] if prefix is not None else 0))
            if window:
                seen &= pos - keys < window
            keys = keys[seen & (keys // page < table.shape[1])]
            at = table[b, keys // page]
            keys, at = keys[(at >= 0) & (at < pages)], at[(at >= 0) & (at < pages)]
            if not len(keys):
                continue
            away = np.abs(pos - keys)
            for g in range(heads):
                k, v = k_cache[at, g // (heads // kv), keys % page], v_cache[at, g // (heads // kv), keys % page]
                z = k @ q[t, g] * scale
                unit[t, g] = (np.abs(k) @ np.abs(q[t, g])).max() * abs(scale)
                if cap:
                    z = cap * np.tanh(z / cap)
                if slopes is not None:
                    z = z - slopes[g] * away
                    unit[t, g] += np.abs(slopes[g] * away).max()
                w = np.exp(z - z.max())
                out[t, g] = w @ v / w.sum()
                size[t, g] = w @ np.abs(v) / w.sum()
                lse[t, g] = z.max() + math.log(w.sum())
    return out, lse, size, unit


def fork(table, lens, parent, keep, num_pages, page):
    """Row by row; shortages and bad values included."""
    n, columns = len(parent), table.shape[1]
    new = np.full((n, columns), -1, np.int64)
    kept = np.zeros(n, np.int64)
    for i, p in enumerate(parent):
        if 0 <= p < len(lens):
            want = lens[p] if keep is None else keep[i]
            kept[i] = want if 0 <= want <= lens[p] and want <= columns * page else 0

    def entry(i, j):
        p = int(table[parent[i], j])
        return p if 0 <= p < num_pages else -1
    shared = set()
    for i in range(n):
        for j in range(kept[i] // page):
            new[i, j] = entry(i, j)
            shared.add(new[i, j])
    owned, source, to, fill = set(), np.full(n, -1, np.int64), np.full(n, -1, np.int64), np.zeros(n, np.int64)
    for i in range(n):
        j = kept[i] // page
        if kept[i] % page and entry(i, j) >= 0:
            p = entry(i, j)
            if p in shared or p in owned:
                source[i], fill[i] = p, kept[i] % page
            else:
                owned.add(p)
                new[i, j] = p
    free = [p for p in range(num_pages) if p not in shared and p not in owned]
    for i in range(n):
        if source[i] >= 0:
            if free:
                to[i] = new[i, kept[i] // page] = free.pop(0)
            else:
                source[i], fill[i] = -1, 0
    return {"table": new, "kv_lens": kept, "copy_from": source, "copy_to": to, "copy_fill": fill,
            "free_pages": np.array(free + [-1] * (num_pages - len(free)), np.int64), "n_free": np.array([len(free)])}


def compact(table, lens, num_pages, page, max_moves):
    n, columns = table.shape
    out = np.full((n, columns), -1, np.int64)
    for b in range(n):
        blocks = min(-(-max(0, int(lens[b])) // page), columns)
        out[b, :blocks] = [p if 0 <= p < num_pages else -1 for p in table[b, :blocks]]
    held = sorted(set(out[out >= 0].tolist()))
    high = [p for p in held if p >= len(held)][::-1]
    low = [p for p in range(len(held)) if p not in set(held)]
    moves = list(zip(high, low))[:max_moves]
    where = dict(moves)
    out = np.array([[where.get(p, p) for p in row] for row in out.tolist()], np.int64).reshape(n, columns)
    pad = [-1] * (max_moves - len(moves))
    return {"table": out, "copy_from": np.array([m[0] for m in moves] + pad, np.int64), "copy_to": np.array([m[1] for m in moves] + pad, np.int64),
            "n_held": np.array([len(held)])}
