"""What is timed of the serving-cache operators: the page map of a step, the norm and rotation of query and key heads
(into a tensor or into the cache, and its gradient), and attention of one new token over the paged cache.

`run` computes them in their plain form, elementary torch operations in 32 bits, or, where `own` is true, through the
library: `prepare` then also binds the operator to its arrays and a scratch buffer, as a serving loop does that runs
one operator on the same arrays every step.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6
THETA = 10000.0
LARGEST_CACHE = 64 * 8192 * 8 * 128       # elements of K that the largest listed attention may read
LARGEST_ROWS = 16384 * 40 * 128           # elements that the largest listed norm and rotation covers


# --------------------------------------------------------------------------- the cases
def listed():
    return [
        # one decoding step of a small server: every request gets one token, now and then a page
        {"name": "pages_step_64", "op": "page_map", "requests": 64, "tokens": 64, "page": 16, "max_len": 4096},
        # a mixed step: some requests leave, half get one token, the rest share the prompts' tokens; odd sizes
        {"name": "pages_mixed_1000", "op": "page_map", "requests": 1000, "tokens": 60013, "page": 48, "max_len": 3000},
        # the largest step: many requests and a million tokens of prompts
        {"name": "pages_prompts_1m", "op": "page_map", "requests": 4096, "tokens": 1 << 20, "page": 64, "max_len": 8192},
        # decoding: the new tokens' heads, keys and values written through the slot map
        {"name": "heads_append_64", "op": "norm_rope", "tokens": 64, "q_heads": 32, "kv_heads": 8, "dim": 128, "rotary": 128,
         "interleaved": False, "axes": 1, "dtype": "bf16", "page": 16},
        # training or a long prompt: all tokens of a batch
        {"name": "heads_train_16k", "op": "norm_rope", "tokens": 16384, "q_heads": 32, "kv_heads": 8, "dim": 128, "rotary": 128,
         "interleaved": False, "axes": 1, "dtype": "bf16", "page": 0},
        # video tokens: three position axes, an odd number of tokens, a narrower head, 16-bit floats
        {"name": "heads_axes_5003", "op": "norm_rope", "tokens": 5003, "q_heads": 12, "kv_heads": 4, "dim": 80, "rotary": 80,
         "interleaved": False, "axes": 3, "dtype": "f16", "page": 0},
        # the gradient of the training case
        {"name": "heads_grad_16k", "op": "norm_rope_grad", "tokens": 16384, "q_heads": 32, "kv_heads": 8, "dim": 128, "rotary": 128,
         "interleaved": False, "axes": 1, "dtype": "bf16", "page": 0},
        # the same in 32 bits for a small model with partly rotated heads, neighbours paired
        {"name": "heads_grad_f32_1237", "op": "norm_rope_grad", "tokens": 1237, "q_heads": 9, "kv_heads": 3, "dim": 64, "rotary": 32,
         "interleaved": True, "axes": 1, "dtype": "f32", "page": 0},
        # a few short conversations: what a call costs
        {"name": "attend_4_short", "op": "attention", "batch": 4, "min_len": 1, "max_len": 300, "q_heads": 8, "kv_heads": 2, "dim": 64,
         "page": 16, "dtype": "f16", "window": 0, "heads_first": False},
        # one long document: the cache's length is all there is to split
        {"name": "attend_1_long", "op": "attention", "batch": 1, "min_len": 131072, "max_len": 131072, "q_heads": 64, "kv_heads": 8, "dim": 128,
         "page": 64, "dtype": "bf16", "window": 0, "heads_first": True},
        # a full server: many requests of every length
        {"name": "attend_64_ragged", "op": "attention", "batch": 64, "min_len": 1, "max_len": 8192, "q_heads": 32, "kv_heads": 8, "dim": 128,
         "page": 16, "dtype": "bf16", "window": 0, "heads_first": False},
        # 32-bit cache, a window, pages that end inside every tile, requests without a token
        {"name": "attend_37_window_f32", "op": "attention", "batch": 37, "min_len": 0, "max_len": 3001, "q_heads": 6, "kv_heads": 6, "dim": 96,
         "page": 24, "dtype": "f32", "window": 1000, "heads_first": True},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["page_map", "norm_rope", "norm_rope_grad", "attention"])
    if op == "page_map":
        requests = _log_uniform(rng, 1, 4096)
        tokens = requests if rng.random() < 0.3 else _log_uniform(rng, requests, 1 << 20)
        return {"op": op, "requests": requests, "tokens": tokens, "page": rng.choice([8, 16, 24, 32, 48, 64, 128]),
                "max_len": _log_uniform(rng, 64, 8192)}
    dim = rng.choice([32, 64, 72, 80, 96, 112, 128, 192, 256])
    kv_heads = _log_uniform(rng, 1, 16)
    q_heads = kv_heads * rng.choice([1, 2, 3, 4, 7, 8, 16])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if op == "attention":
        batch = _log_uniform(rng, 1, 256)
        most = min(131072, LARGEST_CACHE // (batch * kv_heads * dim * (2 if dtype == "f32" else 1)))
        longest = _log_uniform(rng, min(16, most), most)
        return {"op": op, "batch": batch, "min_len": rng.choice([0, 1, longest]), "max_len": longest, "q_heads": q_heads, "kv_heads": kv_heads,
                "dim": dim, "page": rng.choice([1, 8, 16, 24, 32, 48, 64, 128]), "dtype": dtype, "window": rng.choice([0, 0, longest // 3 + 1]),
                "heads_first": rng.random() < 0.5}
    most = min(16384, LARGEST_ROWS // ((q_heads + kv_heads) * dim * (2 if dtype == "f32" else 1)))
    return {"op": op, "tokens": _log_uniform(rng, 1, most), "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "rotary": rng.choice([dim, dim, dim // 2, dim // 4]) // 2 * 2, "interleaved": rng.random() < 0.3, "axes": rng.choice([1, 1, 3]),
            "dtype": dtype, "page": rng.choice([0, 16, 48]) if op == "norm_rope" else 0}


# --------------------------------------------------------------------------- inputs
def _normal(gen, shape, dtype, scale=1.0):
    return torch.randn(shape, dtype=torch.float32, device=DEVICE, generator=gen).mul_(scale).to(dtype)


def _on_device(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEVICE)


def _longest_prompt(case):
    """New tokens of one request at most: four times the mean of the prompts, which half of the requests have."""
    return 1 if case["tokens"] == case["requests"] else 1 + 8 * (case["tokens"] // case["requests"])


def _page_map_arrays(case, seed):
    """The host's view of a step: lengths, new tokens (a request that leaves gives back all it has), pages in use, free pages."""
    rng = np.random.default_rng(seed)
    requests, tokens, page, longest = case["requests"], case["tokens"], case["page"], case["max_len"]
    lengths = np.exp(rng.uniform(0, math.log(longest), requests)).astype(np.int64)
    new = np.ones(requests, np.int64)
    if tokens > requests:
        kind = rng.permutation(requests)
        leaves = kind < requests // 16
        prompts = kind >= requests // 2
        share = rng.random(requests) * prompts
        new = np.where(leaves, -lengths, 1)
        new[prompts] = 1 + np.minimum((tokens - requests) * share[prompts] / share.sum(), _longest_prompt(case) - 1).astype(np.int64)
        lengths[prompts] = np.where(rng.random(requests) < 0.5, 0, lengths)[prompts]       # half of the prompts are new requests
    have = -(-lengths // page)
    need = np.maximum(-(-(lengths + new) // page) - have, 0)
    width = -(-(longest + _longest_prompt(case)) // page)
    pages = requests * -(-longest // page) + tokens // page + requests                     # enough whatever the lengths are
    order = rng.permutation(pages).astype(np.int32)
    table = np.full((requests, width), -1, np.int32)
    in_use = np.arange(width)[None, :] < have[:, None]
    table[in_use] = order[:int(have.sum())]
    free = order[int(have.sum()):][:int(need.sum()) + requests]
    head = int(rng.integers(0, 3 * pages))                                                 # the ring has been round a few times
    pool = np.zeros(pages, np.int32)
    pool[(head + np.arange(free.size)) % pages] = free
    return {"lengths": lengths.astype(np.int32), "new": new.astype(np.int32), "table": table, "pool": pool,
            "cursor": np.array([head, head + free.size], np.int64)}


def _heads_arrays(case, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    t, hq, hk, d, r = (case[k] for k in ("tokens", "q_heads", "kv_heads", "dim", "rotary"))
    dtype = DTYPE[case["dtype"]]
    # one projection's output: queries, keys and values of a token lie side by side
    qkv = _normal(gen, (t, (hq + 2 * hk) * d), dtype, 1.5)
    s = {"q": qkv[:, :hq * d].view(t, hq, d), "k": qkv[:, hq * d:(hq + hk) * d].view(t, hk, d), "v": qkv[:, (hq + hk) * d:].view(t, hk, d),
         "q_weight": (1 + _normal(gen, (d,), torch.float32, 0.2)).to(dtype), "k_weight": (1 + _normal(gen, (d,), torch.float32, 0.2)).to(dtype)}
    furthest = 4096
    s["positions"] = torch.randint(0, furthest, (case["axes"], t), dtype=torch.int32, device=DEVICE, generator=gen)
    angle = torch.arange(furthest, device=DEVICE, dtype=torch.float64)[:, None] * THETA ** (-torch.arange(r // 2, device=DEVICE, dtype=torch.float64) * 2 / r)
    s["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    s["axis_of"] = torch.arange(r // 2, dtype=torch.int32, device=DEVICE) % 3 if case["axes"] == 3 else None
    if case["op"] == "norm_rope_grad":
        s["dq_out"] = _normal(gen, (t, hq, d), dtype)
        s["dk_out"] = _normal(gen, (t, hk, d), dtype)
        s["dq"], s["dk"] = torch.empty_like(s["dq_out"]), torch.empty_like(s["dk_out"])
        s["dq_weight"], s["dk_weight"] = (torch.empty(d, dtype=torch.float32, device=DEVICE) for _ in range(2))
        return s
    s["q_out"] = torch.empty((t, hq, d), dtype=dtype, device=DEVICE)
    if case["page"] == 0:
        s["k_out"] = torch.empty((t, hk, d), dtype=dtype, device=DEVICE)
        return s
    pages = -(-4 * t // case["page"]) + 1
    s["k_cache"] = _normal(gen, (pages, case["page"], hk, d), dtype)
    s["v_cache"] = _normal(gen, (pages, case["page"], hk, d), dtype)
    s["slots"] = torch.randperm(pages * case["page"], device=DEVICE, generator=gen)[:t]
    if t > 8:
        s["slots"][t - t // 8:] = -1                       # the batch is padded: these tokens have no place in the cache
    return s


def _attention_arrays(case, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    b, hq, hk, d, page = (case[k] for k in ("batch", "q_heads", "kv_heads", "dim", "page"))
    dtype = DTYPE[case["dtype"]]
    lengths = np.random.default_rng(seed).integers(case["min_len"], case["max_len"] + 1, b)
    if case["min_len"] == 0:
        lengths[::5] = 0                                   # places of the batch that no request holds
    width = -(-case["max_len"] // page) + 1
    have = -(-lengths // page)
    pages = int(have.sum()) + 3
    table = np.full((b, width), -1, np.int32)
    table[np.arange(width)[None, :] < have[:, None]] = np.random.default_rng(seed + 1).permutation(pages)[:int(have.sum())]
    shape = (pages, hk, page, d) if case["heads_first"] else (pages, page, hk, d)
    k, v = (_normal(gen, shape, dtype) for _ in range(2))
    if case["heads_first"]:
        k, v = k.transpose(1, 2), v.transpose(1, 2)        # [pages, page, heads, dim] whatever the order in memory
    return {"q": _normal(gen, (b, hq, d), dtype, 2.0), "k_cache": k, "v_cache": v, "table": _on_device(table),
            "lengths": _on_device(lengths.astype(np.int32)), "window": case["window"], "longest": case["max_len"],
            "out": torch.empty((b, hq, d), dtype=dtype, device=DEVICE), "lse": torch.empty((b, hq), dtype=torch.float32, device=DEVICE)}


def _operator(case, s):
    """The operator on the state's arrays, as a user of the library describes it."""
    import paper_2407_13585_amd as fc
    if case["op"] == "page_map":
        return fc.PageMap(page_size=case["page"], lengths=s["lengths"], new_tokens=s["new"], pool=s["pool"], cursor=s["cursor"], table=s["table"],
                          lengths_after=s["lengths_after"], row_start=s["row_start"], slots=s["slots"], positions=s["positions"],
                          request=s["request"], cursor_after=s["cursor_after"], unplaced=s["unplaced"])
    if case["op"] == "attention":
        return fc.PagedAttention(q=s["q"], k_cache=s["k_cache"], v_cache=s["v_cache"], table=s["table"], lengths=s["lengths"], out=s["out"],
                                 lse=s["lse"], window=s["window"])
    rotation = {"q_weight": s["q_weight"], "k_weight": s["k_weight"], "eps": EPS, "cos_sin": s["cos_sin"], "positions": s["positions"],
                "axis_of": s["axis_of"], "interleaved": case["interleaved"]}
    if case["op"] == "norm_rope_grad":
        return fc.HeadNormRopeGrad(q=s["q"], k=s["k"], dq_out=s["dq_out"], dk_out=s["dk_out"], dq=s["dq"], dk=s["dk"],
                                   dq_weight=s["dq_weight"], dk_weight=s["dk_weight"], **rotation)
    if case["page"] == 0:
        return fc.HeadNormRope(q=s["q"], k=s["k"], q_out=s["q_out"], k_out=s["k_out"], **rotation)
    return fc.HeadNormRope(q=s["q"], k=s["k"], v=s["v"], q_out=s["q_out"], k_cache=s["k_cache"], v_cache=s["v_cache"], slots=s["slots"], **rotation)


def prepare(case, seed):
    if case["op"] == "page_map":
        s = {k: _on_device(a) for k, a in _page_map_arrays(case, seed).items()}
        b, t = case["requests"], case["tokens"]
        s["lengths_after"], s["row_start"] = (torch.empty(n, dtype=torch.int32, device=DEVICE) for n in (b, b + 1))
        s["positions"], s["request"] = (torch.empty(t, dtype=torch.int32, device=DEVICE) for _ in range(2))
        s["slots"], s["cursor_after"], s["unplaced"] = (torch.empty(n, dtype=torch.int64, device=DEVICE) for n in (t, 2, 1))
    else:
        s = _attention_arrays(case, seed) if case["op"] == "attention" else _heads_arrays(case, seed)
    s["case"] = case
    if own:
        import paper_2407_13585_amd as fc
        operators = [_operator(case, s)]
        s["bound"] = fc.BoundOperators(operators, torch.zeros(fc.fc_operators_scratch_bytes(operators), dtype=torch.uint8, device=DEVICE))
    return s


# --------------------------------------------------------------------------- the plain forms
def _scan(a):
    """Exclusive prefix sums, and the total behind them."""
    return torch.cat([torch.zeros(1, dtype=torch.int64, device=DEVICE), torch.cumsum(a.to(torch.int64), 0)])


def _plain_page_map(s, page):
    pool, table = s["pool"], s["table"]
    requests, width = table.shape
    entries, tokens = pool.numel(), s["slots"].numel()
    length, new = s["lengths"].to(torch.int64).clamp(min=0), s["new"].to(torch.int64)
    head, tail = s["cursor"][0], s["cursor"][1]
    available = (tail - head).clamp(0, entries)
    want = (length + new).clamp(min=0)
    have, goal = (((n + page - 1) // page).clamp(max=width) for n in (length, want))
    need, back = (goal - have).clamp(min=0), (have - goal).clamp(min=0)
    first, behind, row_start = _scan(need), _scan(back), _scan(new.clamp(min=0))
    got = torch.minimum((available - first[:-1]).clamp(min=0), need)
    after = torch.minimum(want, torch.where(new > 0, (have + got) * page, torch.full_like(want, width * page)))
    # new pages out of the ring, given-back ones into it, both over the grid of all entries
    k = torch.arange(width, device=DEVICE)[None, :]
    taken = (k >= have[:, None]) & (k < (have + got)[:, None])
    given = (k >= goal[:, None]) & (k < have[:, None])
    entry = pool[(head + first[:-1, None] + k - have[:, None]) % entries]
    to = torch.where(given, (tail + behind[:-1, None] + k - goal[:, None]) % entries, entries)
    grown = torch.cat([pool, pool[:1]])
    grown[to.reshape(-1)] = torch.where(given, table, table[0, 0]).reshape(-1)
    pool.copy_(grown[:entries])
    table.copy_(torch.where(taken, entry, table))
    # the tokens of the step
    t = torch.arange(tokens, device=DEVICE)
    live = t < row_start[-1]
    r = (torch.searchsorted(row_start, t, right=True) - 1).clamp(max=requests - 1)
    position = length[r] + t - row_start[r]
    at = table.reshape(-1)[r * width + (position // page).clamp(max=width - 1)].to(torch.int64)
    stored = live & (position < after[r]) & (at >= 0)
    s["slots"].copy_(torch.where(stored, at * page + position % page, -1))
    s["positions"].copy_(torch.where(live, position, 0))
    s["request"].copy_(torch.where(live, r, -1))
    s["lengths_after"].copy_(after)
    s["row_start"].copy_(row_start)
    s["cursor_after"].copy_(torch.stack([head + torch.minimum(first[-1], available), tail + behind[-1]]))
    s["unplaced"].copy_((want - after).sum().reshape(1))


def _pairs(x, r, interleaved):
    return (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])


def _unpaired(a, b, rest, interleaved):
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1), rest], -1)


def _angles(s):
    half = s["cos_sin"].shape[1] // 2
    if s["axis_of"] is None:
        row = s["cos_sin"][s["positions"][0]]
        return row[:, None, :half], row[:, None, half:]
    at = s["positions"].t()[:, s["axis_of"]]                                               # a position for each token and pair
    i = torch.arange(half, device=DEVICE)[None, :]
    return s["cos_sin"][at, i][:, None, :], s["cos_sin"][at, half + i][:, None, :]


def _plain_heads(x, weight, cos, sin, interleaved):
    x = x.float()
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    r = 2 * cos.shape[-1]
    a, b = _pairs(y, r, interleaved)
    return _unpaired(a * cos - b * sin, b * cos + a * sin, y[..., r:], interleaved)


def _plain_heads_grad(x, weight, dy, cos, sin, interleaved):
    x, w, dy = x.float(), weight.float(), dy.float()
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    unit = x * rstd
    r = 2 * cos.shape[-1]
    a, b = _pairs(dy, r, interleaved)
    g = _unpaired(a * cos + b * sin, b * cos - a * sin, dy[..., r:], interleaved)
    gw = g * w
    return rstd * (gw - unit * (gw * unit).mean(-1, keepdim=True)), (g * unit).sum((0, 1))


def _plain_attention(s):
    k_cache, v_cache, table = s["k_cache"], s["v_cache"], s["table"]
    batch, hq, d = s["q"].shape
    _, page, hk, _ = k_cache.shape
    n = s["longest"]
    j = torch.arange(n, device=DEVICE)
    length = s["lengths"].to(torch.int64)[:, None]
    live = j < length
    if s["window"]:
        live &= j >= length - s["window"]
    at = table[:, j // page].clamp(min=0).to(torch.int64)
    k, v = (c[at, j % page].transpose(1, 2).float().contiguous() for c in (k_cache, v_cache))       # [batch, heads, n, dim]
    q = s["q"].float().reshape(batch, hk, hq // hk, d)
    live = live[:, None, None, :]
    score = torch.where(live, torch.matmul(q, k.transpose(2, 3).contiguous()) * d ** -0.5, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    s["out"].copy_(o.reshape(batch, hq, d))
    s["lse"].copy_((top + torch.log(total)).reshape(batch, hq))


def _results(case):
    if case["op"] == "page_map":
        return "table", "pool", "lengths_after", "row_start", "slots", "positions", "request", "cursor_after", "unplaced"
    if case["op"] == "attention":
        return "out", "lse"
    if case["op"] == "norm_rope_grad":
        return "dq", "dk", "dq_weight", "dk_weight"
    return ("q_out", "k_cache", "v_cache") if case["page"] else ("q_out", "k_out")


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        s["bound"](torch.cuda.current_stream().cuda_stream)
    elif op == "page_map":
        _plain_page_map(s, case["page"])
    elif op == "attention":
        _plain_attention(s)
    else:
        cos, sin = _angles(s)
        if op == "norm_rope_grad":
            for x in ("q", "k"):
                dx, dw = _plain_heads_grad(s[x], s[x + "_weight"], s[f"d{x}_out"], cos, sin, case["interleaved"])
                s["d" + x].copy_(dx)
                s[f"d{x}_weight"].copy_(dw)
        else:
            s["q_out"].copy_(_plain_heads(s["q"], s["q_weight"], cos, sin, case["interleaved"]))
            k = _plain_heads(s["k"], s["k_weight"], cos, sin, case["interleaved"])
            if case["page"] == 0:
                s["k_out"].copy_(k)
            else:
                # a token without a slot repeats what the first one writes, which always has one
                source = torch.where(s["slots"] >= 0, torch.arange(case["tokens"], device=DEVICE), 0)
                at = s["slots"][source]
                page, offset = at // case["page"], at % case["page"]
                s["k_cache"][page, offset] = k[source].to(s["k_cache"].dtype)
                s["v_cache"][page, offset] = s["v"][source]
    return {name: s[name] for name in _results(case)}


# --------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    if case["op"] == "page_map":
        requests, tokens = case["requests"], case["tokens"]
        new_pages = tokens // case["page"]
        return {"bytes": requests * (4 + 4 + 4 + 4 + 4) + tokens * (8 + 4 + 4) + new_pages * 8 + 40, "flops": 0}
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "attention":
        lengths = np.linspace(case["min_len"], case["max_len"], 1001)                      # uniform between the two, on average
        held = case["batch"] - (-(-case["batch"] // 5) if case["min_len"] == 0 else 0)
        keys = held * float(np.minimum(lengths, case["window"] or case["max_len"]).mean())
        rows = case["batch"] * case["q_heads"]
        return {"bytes": 2 * keys * case["kv_heads"] * case["dim"] * size + rows * (2 * case["dim"] * size + 4) + keys / case["page"] * 4,
                "flops": 4 * keys * case["q_heads"] * case["dim"]}
    t, d = case["tokens"], case["dim"]
    heads = case["q_heads"] + case["kv_heads"]
    angles = min(t, 4096) * case["rotary"] * 4
    if case["op"] == "norm_rope_grad":
        return {"bytes": t * heads * d * size * 3 + angles + t * 4, "flops": t * heads * d * 14}
    values = case["kv_heads"] if case["page"] else 0
    return {"bytes": t * (heads + values) * d * size * 2 + angles + t * 4, "flops": t * heads * d * 8}


# --------------------------------------------------------------------------- from the definitions, in 64 bits
def _exact_page_map(case, seed):
    a = _page_map_arrays(case, seed)
    page, table, pool = case["page"], a["table"], a["pool"]
    width = table.shape[1]
    head, tail = (int(x) for x in a["cursor"])
    free = [int(pool[i % pool.size]) for i in range(head, tail)]
    at, given, start, unplaced = 0, [], [0], 0
    slots, positions, request = (np.full(case["tokens"], fill, np.int64) for fill in (-1, 0, -1))
    after = []
    for r, (length, new) in enumerate(zip(a["lengths"].tolist(), a["new"].tolist())):
        want = max(length + new, 0)
        have, goal = (min(-(-n // page), width) for n in (length, want))
        got = max(min(goal - have, len(free) - at), 0)
        table[r, have:have + got] = free[at:at + got]
        at += got
        given += table[r, goal:have].tolist()
        stored = min(want, (have + got) * page if new > 0 else width * page)
        after.append(stored)
        unplaced += want - stored
        n = max(new, 0)
        p = np.arange(length, length + n)
        here = slice(start[-1], start[-1] + n)
        positions[here], request[here] = p, r
        slots[here] = np.where(p < stored, table[r, np.minimum(p // page, width - 1)].astype(np.int64) * page + p % page, -1)
        start.append(start[-1] + n)
    for i, entry in enumerate(given):
        pool[(tail + i) % pool.size] = entry
    out = {"table": table, "pool": pool, "lengths_after": np.array(after, np.int32), "row_start": np.array(start, np.int32), "slots": slots,
           "positions": positions.astype(np.int32), "request": request.astype(np.int32), "cursor_after": np.array([head + at, tail + len(given)]),
           "unplaced": np.array([unplaced])}
    return {k: torch.from_numpy(v) for k, v in out.items()}


def _exact_rotation(s, r):
    """The rotation of a token's pairs as complex numbers, from the table the operator is given."""
    at = s["positions"].long()
    which = torch.zeros(r // 2, dtype=torch.long, device=DEVICE) if s["axis_of"] is None else s["axis_of"].long()
    i = torch.arange(r // 2, device=DEVICE)
    table = s["cos_sin"].double()
    turn = torch.complex(table[:, :r // 2], table[:, r // 2:])
    return torch.stack([turn[at[which[k]], i[k]] for k in range(r // 2)], 1)[:, None, :]


def _exact_heads(x, weight, turn, interleaved):
    y = weight * x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS)
    r = 2 * turn.shape[-1]
    head = y[..., :r].unflatten(-1, (r // 2, 2)) if interleaved else y[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(head.contiguous()) * turn)
    return torch.cat([(z if interleaved else z.transpose(-1, -2)).flatten(-2), y[..., r:]], -1)


def _exact_attention(case, s):
    page, group, scale = case["page"], case["q_heads"] // case["kv_heads"], 1 / math.sqrt(case["dim"])
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(s["lengths"].tolist()):
        begin = max(0, n - case["window"]) if case["window"] else 0
        if begin == n:
            continue
        first = begin // page
        rows = s["table"][b, first:-(-n // page)].long()
        k, v = (c[rows].flatten(0, 1)[begin - first * page:n - first * page].double().repeat_interleave(group, 1) for c in (s["k_cache"], s["v_cache"]))
        q = s["q"][b].double()
        score = torch.stack([k[:, h] @ q[h] for h in range(q.shape[0])]) * scale
        lse[b] = torch.logsumexp(score, 1)
        p = torch.softmax(score, 1)
        out[b] = torch.stack([p[h] @ v[:, h] for h in range(q.shape[0])])
    return {"out": out, "lse": lse}


def exact(case, seed):
    if case["op"] == "page_map":
        return _exact_page_map(case, seed)
    if case["op"] == "attention":
        return _exact_attention(case, _attention_arrays(case, seed))
    s = _heads_arrays(case, seed)
    turn = _exact_rotation(s, case["rotary"])
    if case["op"] == "norm_rope":
        q, k = (_exact_heads(s[x].double(), s[x + "_weight"].double(), turn, case["interleaved"]) for x in ("q", "k"))
        if case["page"] == 0:
            return {"q_out": q, "k_out": k}
        caches = {}
        for name, rows in (("k_cache", k), ("v_cache", s["v"].double())):
            flat = s[name].double().flatten(0, 1)
            stored = s["slots"] >= 0
            flat[s["slots"][stored]] = rows[stored]
            caches[name] = flat.view(s[name].shape)
        return {"q_out": q, **caches}
    out = {}
    for x in ("q", "k"):
        leaf, weight = (s[n].double().clone().requires_grad_(True) for n in (x, x + "_weight"))
        y = _exact_heads(leaf, weight, turn, case["interleaved"])
        out["d" + x], out[f"d{x}_weight"] = torch.autograd.grad(y, [leaf, weight], s[f"d{x}_out"].double())
    return out
