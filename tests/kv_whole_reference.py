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
    table = np.where((table >= 0) & (table < num_pages), table, -1)
    new = np.full((n, columns), -1, np.int64)
    kept = np.zeros(n, np.int64)
    for i, p in enumerate(parent):
        if 0 <= p < len(lens):
            want = lens[p] if keep is None else keep[i]
            kept[i] = want if 0 <= want <= lens[p] and want <= columns * page else 0
        if kept[i]:
            new[i, : kept[i] // page] = table[p, : kept[i] // page]
    held = np.zeros(num_pages, bool)
    held[new[new >= 0]] = True
    shared = held.copy()
    source, to, fill = np.full(n, -1, np.int64), np.full(n, -1, np.int64), np.zeros(n, np.int64)
    owned = set()
    for i in range(n):
        j = kept[i] // page
        if kept[i] % page and table[parent[i], j] >= 0:
            p = int(table[parent[i], j])
            if shared[p] or p in owned:
                source[i], fill[i] = p, kept[i] % page
            else:
                owned.add(p)
                held[p] = True
                new[i, j] = p
    free = np.flatnonzero(~held)
    taken = 0
    for i in range(n):
        if source[i] >= 0:
            if taken < len(free):
                to[i] = new[i, kept[i] // page] = free[taken]
                taken += 1
            else:
                source[i], fill[i] = -1, 0
    left = free[taken:]
    return {"table": new, "kv_lens": kept, "copy_from": source, "copy_to": to, "copy_fill": fill,
            "free_pages": np.concatenate([left, np.full(num_pages - len(left), -1)]), "n_free": np.array([len(left)])}


def compact(table, lens, num_pages, page, max_moves):
    n, columns = table.shape
    table = np.where((table >= 0) & (table < num_pages), table, -1)
    out = np.full((n, columns), -1, np.int64)
    for b in range(n):
        blocks = min(-(-max(0, int(lens[b])) // page), columns)
        out[b, :blocks] = table[b, :blocks]
    held = np.unique(out[out >= 0])
    high = held[held >= len(held)][::-1][:max_moves]
    low = np.setdiff1d(np.arange(len(held)), held)[:max_moves]
    where = np.concatenate([np.arange(num_pages), [-1]])  # (-1 stays -1)
    where[high] = low
    pad = np.full(max_moves - len(high), -1)
    return {"table": where[out], "copy_from": np.concatenate([high, pad]), "copy_to": np.concatenate([low, pad]), "n_held": np.array([len(held)])}
