"""The operators of a serving cache, from their definitions: numpy, one request / token / head at a time, 64-bit floats.

Test infrastructure only: imports nothing of the package, and the package never imports it.
"""
import numpy as np


def page_map(page_size, lengths, new_tokens, pool, cursor, table, tokens):
    """A step of the page map; the arrays that the operator updates in place are returned as new ones."""
    pool, table = pool.copy(), table.copy()
    width, entries = table.shape[1], pool.size
    head, tail = int(cursor[0]), int(cursor[1])
    available = min(max(tail - head, 0), entries)
    pages = lambda n: min(-(-n // page_size), width)  # noqa: E731
    old, taken, returned, unplaced = pool.copy(), 0, [], 0
    after, start = [], [0]
    request, positions, slots = np.full(tokens, -1, np.int32), np.zeros(tokens, np.int32), np.full(tokens, -1, np.int64)
    for r in range(len(lengths)):
        length, new = max(int(lengths[r]), 0), int(new_tokens[r])
        want = max(length + new, 0)
        have, goal = pages(length), pages(want)
        got = 0
        while have + got < goal and taken < available:
            table[r, have + got] = old[(head + taken) % entries]
            got, taken = got + 1, taken + 1
        returned += [int(p) for p in table[r, goal:have]]
        after.append(min(want, (have + got) * page_size if new > 0 else width * page_size))
        unplaced += want - after[-1]
        for j in range(max(new, 0)):
            t = start[-1] + j
            if t >= tokens:
                break
            request[t], positions[t] = r, length + j
            if length + j < after[-1] and table[r, (length + j) // page_size] >= 0:
                slots[t] = int(table[r, (length + j) // page_size]) * page_size + (length + j) % page_size
        start.append(start[-1] + max(new, 0))
    for i, page in enumerate(returned):
        pool[(tail + i) % entries] = page
    return {"pool": pool, "table": table, "lengths_after": np.array(after, np.int32), "row_start": np.array(start, np.int32), "slots": slots,
            "positions": positions, "request": request, "cursor_after": np.array([head + taken, tail + len(returned)], np.int64),
            "unplaced": np.array([unplaced], np.int64)}


def _pairs(half, interleaved):
    """The two elements of each pair."""
    i = np.arange(half)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + half)


def angles(cos_sin, positions, axis_of):
    """Cosine and sine of each token's pairs: [T, R/2] each; NaN where a position or an axis is outside its table."""
    rows, half = cos_sin.shape[0], cos_sin.shape[1] // 2
    axes, tokens = positions.shape
    c, s = np.full((tokens, half), np.nan), np.full((tokens, half), np.nan)
    for i in range(half):
        axis = 0 if axis_of is None else int(axis_of[i])
        if not (0 <= axis < axes and rows):
            continue
        there = (positions[axis] >= 0) & (positions[axis] < rows)
        at = np.where(there, positions[axis], 0)
        c[there, i], s[there, i] = cos_sin[at, i][there], cos_sin[at, half + i][there]
    return c, s


def turned(y, c, s, interleaved):
    """y [T, H, D] with its first 2 * c.shape[1] elements turned."""
    a, b = _pairs(c.shape[1], interleaved)
    out = y.copy()
    c, s = c[:, None, :], s[:, None, :]
    out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    return out


def head_norm_rope(x, weight, eps, c, s, interleaved):
    """x [T, H, D]; weight None: no norm; c None: no rotation."""
    y = x if weight is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    return y if c is None else turned(y, c, s, interleaved)


def head_norm_rope_grad(x, weight, eps, c, s, interleaved, dy):
    """dx and dweight (None without a weight)."""
    g = dy if c is None else turned(dy, c, -s, interleaved)
    if weight is None:
        return g, None
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u = x * r
    return r * (weight * g - u * (weight * g * u).mean(-1, keepdims=True)), (g * u).sum((0, 1))


def stored(cache, slots, rows):
    """cache [pages, P, H, D] with rows[t] at place slots[t]."""
    cache = cache.copy()
    page = cache.shape[1]
    for t, slot in enumerate(slots):
        if 0 <= slot < cache.shape[0] * page:
            cache[slot // page, slot % page] = rows[t]
    return cache


def paged_attention(q, k_cache, v_cache, table, lengths, scale, window=0):
    """out [B, Hq, D], lse [B, Hq], and what bounds the error of a computation in fewer bits: the largest sum of |q k| scale of a
    query head's keys, and its mean of |v| under the weights."""
    batch, heads, dim = q.shape
    pages, page, kv, _ = k_cache.shape
    out, lse = np.zeros(q.shape), np.full((batch, heads), -np.inf)
    reach, spread = np.zeros((batch, heads)), np.zeros(q.shape)
    for b in range(batch):
        length = max(int(lengths[b]), 0)
        keys = [(int(table[b, j // page]), j % page) for j in range(max(0, length - window) if window else 0, min(length, table.shape[1] * page))]
        keys = [(p, o) for p, o in keys if 0 <= p < pages]
        if not keys:
            continue
        at = np.array(keys)
        for h in range(heads):
            k, v = (cache[at[:, 0], at[:, 1], h // (heads // kv)] for cache in (k_cache, v_cache))
            score = scale * (k @ q[b, h])
            top = score.max()
            p = np.exp(score - top)
            out[b, h], lse[b, h] = p @ v / p.sum(), top + np.log(p.sum())
            reach[b, h], spread[b, h] = abs(scale) * (np.abs(k) @ np.abs(q[b, h])).max(), p @ np.abs(v) / p.sum()
    return out, lse, reach, spread


def page_bounds(k_cache, table, lengths_before, lengths, bounds):
    """bounds [pages, H, 2, D] after a step."""
    bounds = bounds.copy()
    pages, page = k_cache.shape[:2]
    for b in range(len(lengths)):
        before = max(int(lengths_before[b]), 0)
        of_page = {}
        for j in range(before, min(int(lengths[b]), table.shape[1] * page)):
            of_page.setdefault(j // page, []).append(j % page)
        for w, places in of_page.items():
            p = int(table[b, w])
            if not 0 <= p < pages:
                continue
            keys = k_cache[p, places]                        # [new, H, D]
            low, high = keys.min(0), keys.max(0)
            if w * page < before:
                low, high = np.minimum(low, bounds[p, :, 0]), np.maximum(high, bounds[p, :, 1])
            bounds[p, :, 0], bounds[p, :, 1] = low, high
    return bounds


def page_scores(q, bounds):
    """What bounds [n, 2, D] of pages let their keys score with the queries [group, D] of a key head."""
    with np.errstate(invalid="ignore"):
        s = np.array([[(np.maximum(x, 0) * high + np.minimum(x, 0) * low).sum() for x in q] for low, high in bounds])
    return np.where(np.isnan(s), np.inf, s).max(1)


def page_select(q, bounds, table, lengths, page, most, first, last):
    """selected [B, H, most] and the keys selected pages hold [B, H]."""
    batch, width = table.shape
    pages, kv = bounds.shape[:2]
    group = q.shape[1] // kv
    selected, held = np.full((batch, kv, most), -1, np.int32), np.zeros((batch, kv), np.int32)
    for b in range(batch):
        keys = min(max(int(lengths[b]), 0), width * page)
        count = -(-keys // page)
        there = [w for w in range(count) if 0 <= table[b, w] < pages]
        for h in range(kv):
            taken = [w for w in there if w < first or w >= count - last]
            if len(there) <= most:
                taken = there
            else:
                rest = [w for w in there if w not in set(taken)]
                s = page_scores(q[b, h * group:(h + 1) * group], bounds[table[b, rest], h])
                taken = sorted(taken + [rest[i] for i in np.argsort(-s, kind="stable")[:most - len(taken)]])
            selected[b, h, :len(taken)] = table[b, taken]
            held[b, h] = sum(min(page, keys - w * page) for w in taken)
    return selected, held


def attention_of_heads(q, k_cache, v_cache, places, scale):
    """paged_attention where places(b, h) lists the (page, place) that key head h of request b sees; pages outside the cache are left out."""
    batch, heads, _ = q.shape
    pages, _, kv, _ = k_cache.shape
    out, lse = np.zeros(q.shape), np.full((batch, heads), -np.inf)
    reach, spread = np.zeros((batch, heads)), np.zeros(q.shape)
    for b in range(batch):
        for n in range(kv):
            at = np.array([(p, o) for p, o in places(b, n) if 0 <= p < pages], np.int64).reshape(-1, 2)
            if not len(at):
                continue
            k, v = (cache[at[:, 0], at[:, 1], n] for cache in (k_cache, v_cache))
            for h in range(n * (heads // kv), (n + 1) * (heads // kv)):
                score = scale * (k @ q[b, h])
                top = score.max()
                if top == -np.inf:
                    continue
                p = np.exp(score - top)
                out[b, h], lse[b, h] = p @ v / p.sum(), top + np.log(p.sum())
                reach[b, h], spread[b, h] = abs(scale) * (np.abs(k) @ np.abs(q[b, h])).max(), p @ np.abs(v) / p.sum()
    return out, lse, reach, spread


def keys_on(pages, page, length):
    """(page, place) of the first `length` keys on these pages, one after the other."""
    return [(int(pages[j // page]), j % page) for j in range(min(max(int(length), 0), len(pages) * page))]


def selected_attention(q, k_cache, v_cache, table, lengths, scale, window=0):
    """table [B, H, W], lengths [B, H]."""
    page = k_cache.shape[1]
    cut = lambda b, h: max(0, int(lengths[b, h]) - window) if window else 0  # noqa: E731
    return attention_of_heads(q, k_cache, v_cache, lambda b, h: keys_on(table[b, h], page, lengths[b, h])[cut(b, h):], scale)


def prefix_attention(q, k_cache, v_cache, prefix_table, prefix_lengths, group_start, table, lengths, scale):
    page, batch = k_cache.shape[1], len(lengths)
    start = np.maximum.accumulate(np.clip(group_start, 0, batch))
    group = {b: g for g in range(len(prefix_lengths)) for b in range(start[g], start[g + 1])}

    def places(b, h):
        shared = keys_on(prefix_table[group[b]], page, prefix_lengths[group[b]]) if b in group else []
        return shared + keys_on(table[b], page, lengths[b])
    return attention_of_heads(q, k_cache, v_cache, places, scale)
