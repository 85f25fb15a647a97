"""What is timed of the operators that leave most of a long paged cache unread: bounds of a page's keys, attention over the pages
that a score of these bounds selects for each request and key head, and attention of a batch whose requests share a prefix.

`run` computes them in their plain form, elementary torch operations in 32 bits (scores that decide which page is taken in 64), or, where
`own` is true, through the library: `prepare` then also binds the operators to their arrays and a scratch buffer, as a serving loop does
that runs the same ones on the same arrays every step.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
LARGEST_NEW = 65536 * 8 * 128             # elements of new keys that the largest listed bounds cover
LARGEST_CACHE = 64 * 32768 * 8 * 128      # elements of K that the largest listed selection chooses from
LARGEST_SCORES = 64 * 32 * 32768          # scores of queries with a shared prefix
LARGEST_OWN = 200 * 2048 * 8 * 128        # elements of K behind the prefixes


# --------------------------------------------------------------------------- the cases
def listed():
    return [
        # one decoding step of a small server: every request's new key joins the bounds of its last page
        {"name": "bounds_append_64", "op": "bounds", "batch": 64, "tokens": 64, "max_len": 4096, "kv_heads": 8, "dim": 128, "page": 16,
         "dtype": "bf16", "heads_first": False},
        # a step of prompts, pages that are no power of two, an odd number of requests
        {"name": "bounds_prompts_9999", "op": "bounds", "batch": 37, "tokens": 9999, "max_len": 2000, "kv_heads": 3, "dim": 80, "page": 24,
         "dtype": "f32", "heads_first": False},
        # the largest step of prompts
        {"name": "bounds_prompts_64k", "op": "bounds", "batch": 40, "tokens": 65536, "max_len": 4096, "kv_heads": 8, "dim": 128, "page": 32,
         "dtype": "bf16", "heads_first": True},
        # a few short conversations, whose pages are all taken: what the two calls cost
        {"name": "sparse_4_short", "op": "sparse", "batch": 4, "min_len": 1, "max_len": 300, "q_heads": 8, "kv_heads": 2, "dim": 64, "page": 16,
         "pages": 24, "dtype": "f16", "heads_first": False},
        # one long document
        {"name": "sparse_1_long", "op": "sparse", "batch": 1, "min_len": 131072, "max_len": 131072, "q_heads": 64, "kv_heads": 8, "dim": 128,
         "page": 32, "pages": 128, "dtype": "bf16", "heads_first": True},
        # a full server: many requests of every length, each key head reads 2048 keys at most
        {"name": "sparse_64_ragged", "op": "sparse", "batch": 64, "min_len": 1, "max_len": 32768, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "page": 32, "pages": 64, "dtype": "bf16", "heads_first": False},
        # a 32-bit cache, a key head for each query head, pages that end inside every tile, places of the batch that no request holds
        {"name": "sparse_19_f32", "op": "sparse", "batch": 19, "min_len": 0, "max_len": 9001, "q_heads": 6, "kv_heads": 6, "dim": 96, "page": 24,
         "pages": 40, "dtype": "f32", "heads_first": True},
        # four samples of one short question
        {"name": "prefix_4_short", "op": "prefix", "batch": 4, "groups": 1, "loose": 0, "prefix": 500, "own_min": 1, "own_max": 60, "q_heads": 8,
         "kv_heads": 2, "dim": 64, "page": 16, "dtype": "f16", "heads_first": False},
        # many answers about one long document
        {"name": "prefix_64_long", "op": "prefix", "batch": 64, "groups": 1, "loose": 0, "prefix": 32768, "own_min": 1, "own_max": 1000,
         "q_heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "heads_first": False},
        # a server with a system prompt: the requests' own keys are as many as the prompt's
        {"name": "prefix_200_prompt", "op": "prefix", "batch": 200, "groups": 1, "loose": 8, "prefix": 4096, "own_min": 1, "own_max": 2048,
         "q_heads": 32, "kv_heads": 4, "dim": 128, "page": 16, "dtype": "bf16", "heads_first": False},
        # several documents with a few readers each and requests that share nothing, in 32 bits, odd sizes
        {"name": "prefix_37_groups_f32", "op": "prefix", "batch": 37, "groups": 5, "loose": 6, "prefix": 3001, "own_min": 0, "own_max": 500,
         "q_heads": 6, "kv_heads": 6, "dim": 96, "page": 24, "dtype": "f32", "heads_first": True},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["bounds", "sparse", "sparse", "prefix", "prefix"])
    dim = rng.choice([32, 64, 72, 80, 96, 112, 128, 192, 256])
    kv_heads = _log_uniform(rng, 1, 16)
    dtype = rng.choice(["f32", "f16", "bf16"])
    size = 2 if dtype == "f32" else 1
    case = {"op": op, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": rng.choice([8, 16, 24, 32, 48, 64, 128]), "heads_first": rng.random() < 0.5}
    if op == "bounds":
        batch = _log_uniform(rng, 1, 256)
        most = max(batch, LARGEST_NEW // (kv_heads * dim * size))
        tokens = batch if rng.random() < 0.3 else _log_uniform(rng, batch, min(most, 65536))
        return {**case, "batch": batch, "tokens": tokens, "max_len": _log_uniform(rng, 64, min(4096, (1 << 28) // (batch * kv_heads * dim)))}
    q_heads = kv_heads * rng.choice([1, 2, 3, 4, 7, 8, 16])
    if op == "sparse":
        batch = _log_uniform(rng, 1, 128)
        most = min(131072, LARGEST_CACHE // (batch * kv_heads * dim * size))
        longest = _log_uniform(rng, 64, most)
        return {**case, "q_heads": q_heads, "batch": batch, "min_len": rng.choice([0, 1, longest]), "max_len": longest,
                "pages": _log_uniform(rng, 4, 4096 // case["page"] + 4)}
    batch = _log_uniform(rng, 1, 256)
    groups = min(batch, rng.choice([1, 1, 1, 2, 3, 5]))
    most = min(32768, LARGEST_SCORES // (batch * q_heads * groups))
    own_most = min(2048, LARGEST_OWN // (batch * kv_heads * dim * size), 4 * LARGEST_SCORES // (batch * q_heads))
    return {**case, "q_heads": q_heads, "batch": batch, "groups": groups, "loose": (batch - groups) // 8 if rng.random() < 0.5 else 0,
            "prefix": _log_uniform(rng, 16, max(16, most)), "own_min": rng.choice([0, 1]), "own_max": _log_uniform(rng, 1, max(1, own_most))}


# --------------------------------------------------------------------------- inputs
def _normal(gen, shape, dtype, scale=1.0):
    return torch.randn(shape, dtype=torch.float32, device=DEVICE, generator=gen).mul_(scale).to(dtype)


def _on_device(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEVICE)


def _caches(case, gen, pages, count, drift=0.0):
    """`count` caches [pages, page, heads, dim], whatever their order in memory; `drift`: how far the keys of a page are alike."""
    shape = (pages, case["kv_heads"], case["page"], case["dim"]) if case["heads_first"] else (pages, case["page"], case["kv_heads"], case["dim"])
    found = []
    for _ in range(count):
        c = torch.randn(shape, dtype=torch.float32, device=DEVICE, generator=gen)
        if drift:
            places = 2 if case["heads_first"] else 1
            c += drift * torch.randn([1 if k == places else n for k, n in enumerate(shape)], dtype=torch.float32, device=DEVICE, generator=gen)
        c = c.to(DTYPE[case["dtype"]])
        found.append(c.transpose(1, 2) if case["heads_first"] else c)
    return found


def _tables(rng, lists, pages=0):
    """For each (pages of a table, width) a table of pages in random order, -1 behind them; and how many pages there are, `pages` at least."""
    pages = max(pages, sum(int(h.sum()) for h, _ in lists) + 3)
    order, at, tables = rng.permutation(pages).astype(np.int32), 0, []
    for h, width in lists:
        table = np.full((h.size, width), -1, np.int32)
        table[np.arange(width)[None, :] < h[:, None]] = order[at:at + int(h.sum())]
        at += int(h.sum())
        tables.append(table)
    return tables, pages


def _page_bounds(k, count=None):
    """Bounds [pages, heads, 2, dim] of the keys at the first count[page] places of each page (None: all)."""
    k = k.float()
    if count is not None:
        there = (torch.arange(k.shape[1], device=DEVICE)[None, :] < count[:, None])[:, :, None, None]
        low, high = (torch.where(there, k, fill) for fill in (math.inf, -math.inf))
    else:
        low = high = k
    return torch.stack([low.amin(1), high.amax(1)], 2)


def _bounds_arrays(case, seed):
    rng, gen = np.random.default_rng(seed), torch.Generator(DEVICE).manual_seed(seed)
    batch, tokens, page = case["batch"], case["tokens"], case["page"]
    before = np.exp(rng.uniform(0, math.log(case["max_len"]), batch)).astype(np.int64)
    new = np.ones(batch, np.int64)
    if tokens > batch:
        share = rng.random(batch)
        new += ((tokens - batch) * share / share.sum()).astype(np.int64)
        before[rng.random(batch) < 0.5] = 0                # prompts of new requests
    lengths = before + new
    have = -(-lengths // page)
    # as many pages as there can be, whatever the lengths are
    (table,), pages = _tables(rng, [(have, int(have.max()) + 1)], batch * -(-case["max_len"] // page) + tokens // page + 2 * batch)
    k, = _caches(case, gen, pages, 1)
    s = {"k_cache": k, "table": _on_device(table), "before": _on_device(before.astype(np.int32)), "lengths": _on_device(lengths.astype(np.int32))}
    # the bounds that the steps before left: of a page that is begun, of its keys so far; of the others, an earlier request's
    count = np.full(pages, page, np.int64)
    begun = before % page != 0
    count[table[begun, before[begun] // page]] = before[begun] % page
    s["bounds"] = _page_bounds(k, _on_device(count)).to(k.dtype)
    return s


def _sparse_arrays(case, seed):
    rng, gen = np.random.default_rng(seed), torch.Generator(DEVICE).manual_seed(seed)
    b, hq, hk, d, page = (case[k] for k in ("batch", "q_heads", "kv_heads", "dim", "page"))
    lengths = rng.integers(case["min_len"], case["max_len"] + 1, b)
    if case["min_len"] == 0:
        lengths[::5] = 0                                   # places of the batch that no request holds
    have = -(-lengths // page)
    (table,), pages = _tables(rng, [(have, -(-case["max_len"] // page) + 1)])
    k, v = _caches(case, gen, pages, 2, drift=0.5)
    s = {"q": _normal(gen, (b, hq, d), k.dtype, 2.0), "k_cache": k, "v_cache": v, "table": _on_device(table), "lengths": _on_device(lengths.astype(np.int32))}
    # of a page that is not full the bounds of its keys so far
    count = np.full(pages, page, np.int64)
    part = lengths % page != 0
    count[table[part, lengths[part] // page]] = lengths[part] % page
    s["bounds"] = _page_bounds(k, _on_device(count)).to(k.dtype)
    s["selected"] = torch.empty((b, hk, case["pages"]), dtype=torch.int32, device=DEVICE)
    s["selected_lengths"] = torch.empty((b, hk), dtype=torch.int32, device=DEVICE)
    return s


def _prefix_arrays(case, seed):
    rng, gen = np.random.default_rng(seed), torch.Generator(DEVICE).manual_seed(seed)
    b, groups, hq, d, page = (case[k] for k in ("batch", "groups", "q_heads", "dim", "page"))
    cuts = np.sort(rng.permutation(b - case["loose"] - 1)[:groups - 1] + 1)                # each group has a request at least
    first = case["loose"] // 2                             # requests without a prefix lie on both sides
    start = np.concatenate([[0], cuts, [b - case["loose"]]]) + first
    prefix = rng.integers((case["prefix"] + 1) // 2, case["prefix"] + 1, groups)
    prefix[0] = case["prefix"]
    lengths = rng.integers(case["own_min"], case["own_max"] + 1, b)
    have = [-(-n // page) for n in (prefix, lengths)]
    (prefix_table, table), pages = _tables(rng, [(have[0], int(have[0].max()) + 1), (have[1], -(-case["own_max"] // page) + 1)])
    k, v = _caches(case, gen, pages, 2)
    return {"q": _normal(gen, (b, hq, d), k.dtype, 2.0), "k_cache": k, "v_cache": v, "prefix_table": _on_device(prefix_table),
            "prefix_lengths": _on_device(prefix.astype(np.int32)), "group_start": _on_device(start.astype(np.int32)), "table": _on_device(table),
            "lengths": _on_device(lengths.astype(np.int32)), "longest_prefix": case["prefix"], "longest": case["own_max"], "largest_group": int(np.diff(start).max())}


ARRAYS = {"bounds": _bounds_arrays, "sparse": _sparse_arrays, "prefix": _prefix_arrays}


def _operators(case, s):
    """The operators on the state's arrays, as a user of the library describes them."""
    import paper_2407_13585_amd as fc
    if case["op"] == "bounds":
        return [fc.PageBounds(k_cache=s["k_cache"], table=s["table"], lengths_before=s["before"], lengths=s["lengths"], bounds=s["bounds"])]
    cache = {"q": s["q"], "k_cache": s["k_cache"], "v_cache": s["v_cache"], "out": s["out"], "lse": s["lse"]}
    if case["op"] == "sparse":
        return [fc.PageSelect(q=s["q"], bounds=s["bounds"], table=s["table"], lengths=s["lengths"], page_size=case["page"], first=1, last=2,
                              selected=s["selected"], selected_lengths=s["selected_lengths"]),
                fc.PagedAttention(table=s["selected"], lengths=s["selected_lengths"], **cache)]
    return [fc.PrefixAttention(prefix_table=s["prefix_table"], prefix_lengths=s["prefix_lengths"], group_start=s["group_start"], table=s["table"],
                               lengths=s["lengths"], **cache)]


def prepare(case, seed):
    s = ARRAYS[case["op"]](case, seed)
    if case["op"] != "bounds":
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEVICE)
    s["case"] = case
    if own:
        import paper_2407_13585_amd as fc
        operators = _operators(case, s)
        s["bound"] = fc.BoundOperators(operators, torch.zeros(fc.fc_operators_scratch_bytes(operators), dtype=torch.uint8, device=DEVICE))
    return s


# --------------------------------------------------------------------------- the plain forms
def _plain_bounds(s, page):
    k, table, bounds = s["k_cache"], s["table"], s["bounds"]
    at = torch.arange(table.shape[1], device=DEVICE)[None, :]
    before, after = s["before"].to(torch.int64)[:, None], s["lengths"].to(torch.int64)[:, None]
    touched = (at * page < after) & ((at + 1) * page > before)
    request, place = touched.nonzero(as_tuple=True)
    of = table[request, place].to(torch.int64)
    position = place[:, None] * page + torch.arange(page, device=DEVICE)
    new = ((position >= before[request]) & (position < after[request]))[:, :, None, None]
    keys = k[of].float()
    low, high = torch.where(new, keys, math.inf).amin(1), torch.where(new, keys, -math.inf).amax(1)
    begun = (place * page < before[request, 0])[:, None, None]
    old = bounds[of].float()
    low = torch.where(begun, torch.minimum(low, old[:, :, 0]), low)
    high = torch.where(begun, torch.maximum(high, old[:, :, 1]), high)
    bounds[of] = torch.stack([low, high], 2).to(bounds.dtype)


def _plain_select(s, page, first, last):
    """The pages that count most for each request and key head, in order; ties go to the lower position."""
    table, bounds, selected = s["table"], s["bounds"], s["selected"]
    batch, width = table.shape
    hk, most = selected.shape[1:]
    length = s["lengths"].to(torch.int64)[:, None]
    pages = (length + page - 1) // page
    at = torch.arange(width, device=DEVICE)[None, :]
    live = (at < pages) & (table >= 0) & (table < bounds.shape[0])
    of = bounds[torch.where(live, table, 0).to(torch.int64)].double()                      # [batch, width, heads, 2, dim]
    q = s["q"].double().reshape(batch, hk, -1, s["q"].shape[-1])
    signed = torch.cat([q.clamp(max=0), q.clamp(min=0)], -1)
    score = torch.matmul(signed, of.flatten(3).permute(0, 2, 3, 1).contiguous())           # [batch, heads, group, width]
    score = torch.where(score.isnan(), math.inf, score).amax(2)
    always = live & ((at < first) | (at >= pages - last))
    # what is always taken stands before all scores, what is not there behind them
    rank = torch.where(always, 2, torch.where(live, 1, 0))[:, None, :].expand(batch, hk, width)
    order = torch.sort(score, dim=2, descending=True, stable=True).indices
    order = order.gather(2, torch.sort(rank.gather(2, order), dim=2, descending=True, stable=True).indices)[:, :, :most]
    taken = rank.gather(2, order) > 0
    order = torch.sort(torch.where(taken, order, width), dim=2).values
    taken = order < width
    short = torch.full((batch, hk, most - order.shape[2]), width, device=DEVICE) if most > order.shape[2] else order[:, :, :0]
    order, taken = torch.cat([order, short], 2), torch.cat([taken, short < width], 2)
    entry = table[:, None, :].expand(batch, hk, width).gather(2, order.clamp(max=width - 1))
    selected.copy_(torch.where(taken, entry, -1))
    missing = torch.where(order == pages[:, None] - 1, pages[:, None] * page - length[:, None], 0).sum(2)
    s["selected_lengths"].copy_(taken.sum(2) * page - missing)


def _rows(cache, table, n):
    """The first n positions of each table, [.., n, dim] in 32 bits: of all heads, [tables, heads, n, dim], or of each head's own table."""
    page = cache.shape[1]
    j = torch.arange(n, device=DEVICE)
    at = table[..., j // page].clamp(min=0).to(torch.int64)
    if table.dim() == 2:
        return cache[at, j % page].transpose(1, 2).float().contiguous()
    return cache[at, j % page, torch.arange(table.shape[1], device=DEVICE)[None, :, None]].float()


def _scores(q, k, n, scale):
    """Scores of q [.., heads, rows, dim] with the first n [..] keys of k, -inf behind them."""
    live = torch.arange(k.shape[-2], device=DEVICE) < n[..., None]
    return torch.where(live[..., None, :], torch.matmul(q, k.transpose(-1, -2).contiguous()) * scale, -math.inf)


def _weights(score, top):
    return torch.exp(score - torch.where(top == -math.inf, 0.0, top))


def _plain_sparse(s, page):
    _plain_select(s, page, 1, 2)
    batch, hq, d = s["q"].shape
    hk, most = s["selected"].shape[1:]
    k, v = (_rows(c, s["selected"], most * page) for c in (s["k_cache"], s["v_cache"]))
    score = _scores(s["q"].float().reshape(batch, hk, hq // hk, d), k, s["selected_lengths"], d ** -0.5)
    top = score.amax(-1, keepdim=True)
    p = _weights(score, top)
    total = p.sum(-1, keepdim=True)
    s["out"].copy_((torch.matmul(p, v) / torch.where(total > 0, total, 1.0)).reshape(batch, hq, d))
    s["lse"].copy_((top + torch.log(total)).reshape(batch, hq))


def _plain_prefix(s):
    batch, hq, d = s["q"].shape
    hk = s["k_cache"].shape[2]
    scale, group = d ** -0.5, hq // hk
    q = s["q"].float().reshape(batch, hk, group, d)
    start = s["group_start"].to(torch.int64)
    groups, members = start.numel() - 1, s["largest_group"]
    # the requests of each group side by side, every key of its prefix read once for all of them
    member = start[:-1, None] + torch.arange(members, device=DEVICE)
    there = member < start[1:, None]
    member = torch.where(there, member, 0)
    shared = q[member].permute(0, 2, 1, 3, 4).reshape(groups, hk, members * group, d)
    k, v = (_rows(c, s["prefix_table"], s["longest_prefix"]) for c in (s["k_cache"], s["v_cache"]))
    score = _scores(shared, k, s["prefix_lengths"][:, None].expand(groups, hk), scale)
    top_shared = score.amax(-1, keepdim=True)
    p = _weights(score, top_shared)
    of_group = torch.cat([p.sum(-1, keepdim=True), top_shared, torch.matmul(p, v)], -1).reshape(groups, hk, members, group, d + 2).transpose(1, 2)
    # back to the order of the batch; a request of no group has seen nothing
    state = torch.zeros((batch + 1, hk, group, d + 2), device=DEVICE)
    state[..., 1] = -math.inf
    state[torch.where(there, member, batch)] = of_group.contiguous()
    total_shared, top_shared, sum_shared = state[:batch, ..., :1], state[:batch, ..., 1:2], state[:batch, ..., 2:]
    k, v = (_rows(c, s["table"], s["longest"]) for c in (s["k_cache"], s["v_cache"]))
    score = _scores(q, k, s["lengths"][:, None].expand(batch, hk), scale)
    top_own = score.amax(-1, keepdim=True)
    p = _weights(score, top_own)
    top = torch.maximum(top_own, top_shared)
    f_own, f_shared = _weights(top_own, top), _weights(top_shared, top)
    total = p.sum(-1, keepdim=True) * f_own + total_shared * f_shared
    o = (torch.matmul(p, v) * f_own + sum_shared * f_shared) / torch.where(total > 0, total, 1.0)
    s["out"].copy_(o.reshape(batch, hq, d))
    s["lse"].copy_((top + torch.log(total)).reshape(batch, hq))


RESULTS = {"bounds": ("bounds",), "sparse": ("selected", "selected_lengths", "out", "lse"), "prefix": ("out", "lse")}


def run(s):
    case = s["case"]
    if own:
        s["bound"](torch.cuda.current_stream().cuda_stream)
    elif case["op"] == "bounds":
        _plain_bounds(s, case["page"])
    elif case["op"] == "sparse":
        _plain_sparse(s, case["page"])
    else:
        _plain_prefix(s)
    return {name: s[name] for name in RESULTS[case["op"]]}


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    hk, d, page, batch = case["kv_heads"], case["dim"], case["page"], case["batch"]
    if case["op"] == "bounds":
        pages = min(case["tokens"], case["tokens"] / page + batch)                         # touched, on average nearly
        begun = batch if case["tokens"] == batch else batch / 2
        return {"bytes": case["tokens"] * hk * d * size + (pages + begun) * 2 * hk * d * size + pages * 4 + batch * 8, "flops": 2 * case["tokens"] * hk * d}
    hq = case["q_heads"]
    rows = batch * hq * (2 * d * size + 4)
    if case["op"] == "sparse":
        held = batch - (-(-batch // 5) if case["min_len"] == 0 else 0)
        lengths = np.linspace(case["min_len"], case["max_len"], 1001)                      # uniform between the two, on average
        pages = held * float(np.ceil(lengths / page).mean())
        keys = held * float(np.minimum(lengths, case["pages"] * page).mean())
        return {"bytes": pages * (2 * hk * d * size + 4) + 2 * keys * hk * d * size + rows + batch * hk * (case["pages"] + 1) * 4,
                "flops": 4 * pages * hq * d + 4 * keys * hq * d}
    keys = case["prefix"] * (1 + 0.75 * (case["groups"] - 1))
    seen = (batch - case["loose"]) * keys / case["groups"]
    own_keys = batch * (case["own_min"] + case["own_max"]) / 2
    return {"bytes": 2 * (keys + own_keys) * hk * d * size + rows + (keys + own_keys) / page * 4, "flops": 4 * (seen + own_keys) * hq * d}


# --------------------------------------------------------------------------- from the definitions, in 64 bits
def _exact_bounds(case, s):
    page, bounds = case["page"], s["bounds"].double().clone()
    k = s["k_cache"].double()
    table = s["table"].tolist()
    for b, (n, m) in enumerate(zip(s["before"].tolist(), s["lengths"].tolist())):
        for w in range(n // page, -(-m // page)):
            lo, hi = max(n - w * page, 0), min(m - w * page, page)
            of = table[b][w]
            low, high = k[of, lo:hi].min(0).values, k[of, lo:hi].max(0).values
            if lo:
                low, high = torch.minimum(low, bounds[of, :, 0]), torch.maximum(high, bounds[of, :, 1])
            bounds[of, :, 0], bounds[of, :, 1] = low, high
    return {"bounds": bounds}


def _exact_heads(q, keys, values, scale):
    """out [rows, dim] and lse [rows] of queries [rows, dim] over keys [n, dim]."""
    score = (q @ keys.t()) * scale
    return torch.softmax(score, -1) @ values, torch.logsumexp(score, -1)


def _exact_sparse(case, s):
    page, most, hk, d = case["page"], case["pages"], case["kv_heads"], case["dim"]
    group = case["q_heads"] // hk
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEVICE)
    selected, lengths = np.full((case["batch"], hk, most), -1, np.int32), np.zeros((case["batch"], hk), np.int32)
    for b, n in enumerate(s["lengths"].tolist()):
        if n == 0:
            continue
        count = -(-n // page)
        of = s["table"][b, :count].long()
        for h in range(hk):
            q = s["q"][b, h * group:(h + 1) * group].double()
            low, high = s["bounds"][of, h, 0].double(), s["bounds"][of, h, 1].double()
            # the larger of the two products in every dimension
            score = torch.stack([torch.maximum(x * low, x * high).sum(1) for x in q]).amax(0).cpu().numpy()
            taken = {0, count - 1, max(count - 2, 0)}
            for at in sorted(range(count), key=lambda w: (-score[w], w)):
                if len(taken) >= most:
                    break
                taken.add(at)
            chosen = sorted(taken)
            rows = torch.tensor(chosen, device=DEVICE)
            selected[b, h, :len(chosen)] = of[rows].cpu().numpy()
            live = len(chosen) * page - (count * page - n)
            lengths[b, h] = live
            k, v = (c[of[rows], :, h].double().flatten(0, 1)[:live] for c in (s["k_cache"], s["v_cache"]))
            out[b, h * group:(h + 1) * group], lse[b, h * group:(h + 1) * group] = _exact_heads(q, k, v, 1 / math.sqrt(d))
    return {"selected": torch.from_numpy(selected), "selected_lengths": torch.from_numpy(lengths), "out": out, "lse": lse}


def _exact_prefix(case, s):
    page, hk, d = case["page"], case["kv_heads"], case["dim"]
    group = case["q_heads"] // hk
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEVICE)

    def rows(table, n):
        of = table[:-(-n // page)].long()
        return [c[of].flatten(0, 1)[:n].double().transpose(0, 1).contiguous() for c in (s["k_cache"], s["v_cache"])]
    start, lengths = s["group_start"].tolist(), s["lengths"].tolist()
    of_group = {b: g for g in range(case["groups"]) for b in range(start[g], start[g + 1])}
    shared = [rows(s["prefix_table"][g], n) for g, n in enumerate(s["prefix_lengths"].tolist())]
    for b in range(case["batch"]):
        parts = [rows(s["table"][b], lengths[b])] + ([shared[of_group[b]]] if b in of_group else [])
        if sum(p[0].shape[1] for p in parts) == 0:
            continue
        k, v = (torch.cat([p[i] for p in parts], 1) for i in range(2))
        q = s["q"][b].double().reshape(hk, group, d)
        score = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(d)
        out[b] = torch.matmul(torch.softmax(score, -1), v).reshape(-1, d)
        lse[b] = torch.logsumexp(score, -1).reshape(-1)
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = ARRAYS[case["op"]](case, seed)
    return {"bounds": _exact_bounds, "sparse": _exact_sparse, "prefix": _exact_prefix}[case["op"]](case, s)
