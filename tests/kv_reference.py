"""Plain 64-bit forms of the block-cache operators, written from their formulas in numpy.  Nothing here is shared
with the library; where a definition rounds to 32 bits (summary codes, scores) the rounding is done here too."""
import math

import numpy as np

UNIT = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}  # largest relative rounding error of the type
TINY = {"bf16": 1e-38, "fp16": 2.0 ** -25}      # largest absolute one among its smallest numbers


def ceil_div(a, b):
    return -(-a // b)


def tables(cached, fresh, page, free, table, max_tokens, max_touched):
    """Sequential restatement; shortages and bad lengths included."""
    table = table.astype(np.int64).copy()
    n, columns = table.shape
    out = {"kv_lens": [], "token_start": [0], "used": 0}
    req, pos, slot, tpage, tfill = [], [], [], [], []
    for b in range(n):
        c, f = int(cached[b]), int(fresh[b])
        if c < 0 or f < 0:
            c = f = 0
        old, now = ceil_div(c, page), ceil_div(c + f, page)
        row = [int(table[b, j]) if j < columns else -1 for j in range(old)]
        for j in range(old, now):
            take = out["used"]
            out["used"] += 1
            row.append(int(free[take]) if take < len(free) and j < columns else -1)
        for j in range(old, columns):
            table[b, j] = row[j] if j < now else -1
        for i in range(f):
            p = c + i
            req.append(b)
            pos.append(p)
            at = row[p // page]
            slot.append(at * page + p % page if at >= 0 else -1)
        if f:
            for j in range(c // page, now):
                tpage.append(row[j])
                tfill.append(min(page, c + f - j * page) if row[j] >= 0 else 0)
        out["kv_lens"].append(c + f)
        out["token_start"].append(out["token_start"][-1] + f)

    def padded(a, size, with_):
        return np.array((a + [with_] * size)[:size], np.int64)
    out.update(table=table, token_req=padded(req, max_tokens, -1), token_pos=padded(pos, max_tokens, -1), token_slot=padded(slot, max_tokens, -1),
               touched_page=padded(tpage, max_touched, -1), touched_fill=padded(tfill, max_touched, 0))
    return out


def turned(x, weight, eps, rotary, pos, interleaved):
    """Norm and rotation of [n, heads, d] float64 rows, and the sum of magnitudes in each output (for tolerances)."""
    y = x.copy()
    if weight is not None:
        y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps) * weight
    size = np.abs(y)
    rot = 0 if rotary is None else rotary.shape[1]
    out, mag = y.copy(), size.copy()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        c, s = rotary[pos, i][:, None], rotary[pos, rot // 2 + i][:, None]
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., a] * s + y[..., b] * c
        mag[..., a] = mag[..., b] = size[..., a] + size[..., b]
    return out, mag


def halved(x):
    x = x.astype(np.float32)
    n = 1 << (x.shape[0] - 1).bit_length()
    x = np.concatenate([x, np.zeros((n - x.shape[0],) + x.shape[1:], np.float32)])
    while x.shape[0] > 1:
        x = x[: x.shape[0] // 2] + x[x.shape[0] // 2:]
    return x[0]


def coded(x):
    """(codes, scale) of rows of float32."""
    scale = np.abs(x).max(-1) * np.float32(1.0 / 127)
    scale = np.where(scale >= np.float32(2.0 ** -126), scale, np.float32(0))
    unit = np.where(scale > 0, scale, np.float32(1))[..., None]
    codes = np.clip(np.rint(x / unit), -127, 127)
    return np.where(scale[..., None] > 0, codes, 0).astype(np.int64), scale


def summary(keys, fill):
    """(codes, scales, mean in 64 bits) of one page's keys [heads, page, d]."""
    x = keys[:, :fill].astype(np.float32).transpose(1, 0, 2)
    pad = np.zeros((keys.shape[1] - fill,) + x.shape[1:], np.float32)
    mean = halved(np.concatenate([x, pad])) / np.float32(fill)
    codes, scale = coded(mean)
    return codes, scale, keys[:, :fill].mean(1)


def select(q, codes, scales, table, req, pos, page, take, n_first, n_last):
    n, heads, d = q.shape
    kv = codes.shape[1]
    out = np.full((n, kv, take), -1, np.int64)
    for t in range(n):
        if req[t] < 0 or pos[t] < 0:
            continue
        last = pos[t] // page
        for h in range(kv):
            u, _ = coded(halved(q[t, h * (heads // kv): (h + 1) * (heads // kv)]))
            rated = []
            for b in range(last + 1):
                p = table[req[t], b]
                if not 0 <= p < codes.shape[0]:
                    continue
                score = np.float32(np.float64(int((u * codes[p, h]).sum())) * np.float64(scales[p, h]))
                rated.append((-math.inf if b < n_first or b > last - n_last else -score, b))
            best = sorted(b for _, b in sorted(rated)[:take])
            out[t, h, : len(best)] = best
    return out


def attend(q, k_cache, v_cache, table, req, pos, selected, scale):
    """(out, lse, attention-weighted mean of |v|, largest logit error unit): caches [pages, kv_heads, page, d], float64."""
    n, heads, d = q.shape
    kv, page = k_cache.shape[1:3]
    group = heads // kv
    out, size = np.zeros((n, heads, d)), np.zeros((n, heads, d))
    lse, unit = np.full((n, heads), -np.inf), np.zeros((n, heads))
    for t in range(n):
        if req[t] < 0 or pos[t] < 0:
            continue
        for h in range(kv):
            at = [(table[req[t], b], o) for b in selected[t, h] if b >= 0 for o in range(page) if b * page + o <= pos[t]]
            if not at:
                continue
            p, o = np.array(at).T
            k, v = k_cache[p, h, o], v_cache[p, h, o]
            for g in range(h * group, (h + 1) * group):
                z = k @ q[t, g] * scale
                w = np.exp(z - z.max())
                out[t, g] = w @ v / w.sum()
                size[t, g] = w @ np.abs(v) / w.sum()
                lse[t, g] = z.max() + math.log(w.sum())
                unit[t, g] = (np.abs(k) @ np.abs(q[t, g])).max() * abs(scale)
    return out, lse, size, unit
