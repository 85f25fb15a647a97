"""The operators of a serving cache on the GPU against the definitions in 64 bits (oracle/cache.py).

Tolerances.  u = 2^-24, 2^-11, 2^-8: unit roundoff of f32, f16, bf16, which a result is rounded to once; `tiny`: half the spacing of
the smallest f16 numbers.  Everything before that is in 32 bits:
  * norm: a sum of at most 512 squares in a tree of at most 22 roundings, halved by the root, 5 more: 16 * 2^-24 |y|; the rotation
    adds two products and a sum: 20 * 2^-24 (|a| + |b|).
  * gradient: the same for dx = r (gw - x mean(gw x)) with the terms' magnitudes; the weights' gradients are sums of tokens * heads
    terms in a fixed tree: 1e-5 of the sum of magnitudes, as for every sum of this library.
  * attention: a score is a sum of D products: (D + 8) * 2^-24 of the sum of magnitudes, `e`.  The weights follow with relative error
    e + 2^-20, held in at least 16 bits (2^-16): twice that, once in the sum above and once in the one below, of the mean of |v|.
"""
import math

import numpy as np
import pytest

from oracle import cache as O

pytestmark = pytest.mark.gpu

U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -25, "bf16": 1e-37}


def types():
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def gpu(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(types()[dtype])


def host(t):
    """On the host, floats in 64 bits."""
    t = t.detach().cpu()
    return t.double().numpy() if t.is_floating_point() else t.numpy()


def run(ops, stream=None, repeat=1):
    import torch
    import paper_2407_13585_amd as fc
    scratch = torch.zeros(fc.fc_operators_scratch_bytes(ops), dtype=torch.uint8, device="cuda")
    for _ in range(repeat):
        fc.fc_run_operators(ops, scratch, (stream or torch.cuda.current_stream()).cuda_stream)
    torch.cuda.synchronize()


def near(got, want, tol, what=""):
    """Finite values within tol, the others the same."""
    got, tol = np.asarray(got, np.float64), np.broadcast_to(tol, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine), f"{what}: not finite on one side only"
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True), what
    err = np.abs(got[fine] - want[fine])
    if err.size and not np.all(err <= tol[fine]):
        i = int(np.argmax(err / np.maximum(tol[fine], 1e-300)))
        raise AssertionError(f"{what}: {got[fine][i]!r} is not {want[fine][i]!r}: off by {err[i]:.3g}, {tol[fine][i]:.3g} allowed")


# --------------------------------------------------------------------------- page map
def map_case(requests, page, longest, seed, kind="mixed", width=None, tokens=None, spare=5, short=0):
    """lengths, new tokens, a table whose pages are in use, and a ring that has been round a few times.  short: pages the ring lacks."""
    rng = np.random.default_rng(seed)
    lengths = rng.integers(0, longest + 1, requests)
    if kind == "step":
        new = np.ones(requests, np.int64)
    elif kind == "nothing":
        new = np.zeros(requests, np.int64)
    else:
        new = np.where(rng.random(requests) < 0.3, rng.integers(0, longest + 1, requests), rng.integers(-longest, 3, requests))
        new[rng.random(requests) < 0.2] = 0
        leaves = rng.random(requests) < 0.2
        new[leaves] = -lengths[leaves]
    width = width or -(-2 * longest // page) + 2
    pages = lambda n: np.minimum(-(-n // page), width)  # noqa: E731
    have = pages(lengths)
    need = np.maximum(pages(np.maximum(lengths + new, 0)) - have, 0)
    free = max(int(need.sum()) + spare - short, 0)
    order = rng.permutation(int(have.sum()) + free).astype(np.int32)
    table = np.full((requests, width), -7, np.int32)
    table[np.arange(width)[None, :] < have[:, None]] = order[:have.sum()]
    entries = order.size
    head = int(rng.integers(0, 5 * max(entries, 1)))
    pool = np.full(entries, -9, np.int32)
    if entries:
        pool[(head + np.arange(free)) % entries] = order[have.sum():]
    total = int(np.maximum(new, 0).sum())
    return dict(page_size=page, lengths=lengths.astype(np.int32), new_tokens=new.astype(np.int32), pool=pool,
                cursor=np.array([head, head + free], np.int64), table=table, tokens=total + 3 if tokens is None else tokens)


def check_map(case, repeat=1, table_room=0):
    import torch
    import paper_2407_13585_amd as fc
    want = O.page_map(**case)
    requests, width = case["table"].shape
    held = torch.full((requests, width + table_room), 12345, dtype=torch.int32, device="cuda")
    table = held[:, :width]
    table.copy_(gpu(case["table"]))
    ins = {k: gpu(case[k]) for k in ("lengths", "new_tokens", "pool", "cursor")}
    i32, i64 = torch.int32, torch.int64
    outs = {k: torch.full((n,), -77, dtype=t, device="cuda") for k, n, t in (
        ("lengths_after", requests, i32), ("row_start", requests + 1, i32), ("slots", case["tokens"], i64), ("positions", case["tokens"], i32),
        ("request", case["tokens"], i32), ("cursor_after", 2, i64), ("unplaced", 1, i64))}
    run([fc.PageMap(page_size=case["page_size"], table=table, **ins, **outs)], repeat=repeat)
    for name, t in {"pool": ins["pool"], "table": table, **outs}.items():
        assert np.array_equal(host(t), want[name]), name
    for name in ("lengths", "new_tokens", "cursor"):
        assert np.array_equal(host(ins[name]), case[name]), name
    assert (held[:, width:] == 12345).all()
    return want


def check_map_counted(case):
    """The same where the oracle would count one by one and its row_start would not fit: computed on fewer tokens, with the same pages."""
    import torch
    import paper_2407_13585_amd as fc
    size = 1 << 20                                              # the oracle's pages are that much smaller
    small = {**case, "page_size": case["page_size"] // size, "lengths": -(-case["lengths"].astype(np.int64) // size),
             "new_tokens": -(-(case["lengths"].astype(np.int64) + case["new_tokens"]) // size) - -(-case["lengths"].astype(np.int64) // size)}
    want = O.page_map(**small)
    requests = len(case["lengths"])
    ins = {k: gpu(case[k]) for k in ("lengths", "new_tokens", "pool", "cursor", "table")}
    outs = {k: torch.full((n,), -77, dtype=t, device="cuda") for k, n, t in (
        ("lengths_after", requests, torch.int32), ("row_start", requests + 1, torch.int32), ("slots", case["tokens"], torch.int64),
        ("positions", case["tokens"], torch.int32), ("request", case["tokens"], torch.int32), ("cursor_after", 2, torch.int64), ("unplaced", 1, torch.int64))}
    run([fc.PageMap(page_size=case["page_size"], **ins, **outs)])
    assert np.array_equal(host(ins["table"]), want["table"]) and np.array_equal(host(ins["pool"]), want["pool"])
    assert np.array_equal(host(outs["cursor_after"]), want["cursor_after"])
    sums = np.concatenate([[0], np.cumsum(case["new_tokens"].astype(np.int64))])
    assert np.array_equal(host(outs["row_start"]), np.minimum(sums, 2 ** 31 - 1))
    whole = case["lengths"].astype(np.int64) + case["new_tokens"]
    held = (want["table"] >= 0).sum(1).astype(np.int64) * case["page_size"]
    assert np.array_equal(host(outs["lengths_after"]), np.minimum(whole, held)) and host(outs["unplaced"])[0] == (whole - np.minimum(whole, held)).sum()
    first = np.arange(case["tokens"]) + case["lengths"][0]
    assert np.array_equal(host(outs["positions"]), first) and (host(outs["request"]) == 0).all()
    assert np.array_equal(host(outs["slots"]), want["table"][0][first // case["page_size"]].astype(np.int64) * case["page_size"] + first % case["page_size"])
    return want


@pytest.mark.parametrize("requests", [1, 2, 63, 64, 65, 257, 1000, 1025, 4095, 4096, 4097, 9001])
@pytest.mark.parametrize("kind", ["step", "mixed"])
def test_page_map_of_many_and_few_requests(requests, kind):
    check_map(map_case(requests, 16, 70 if requests > 500 else 300, seed=requests, kind=kind))


@pytest.mark.parametrize("page", [1, 3, 7, 16, 24, 1000])
def test_page_map_with_pages_of_any_size(page):
    for seed in range(4):
        check_map(map_case(37, page, 131, seed=100 * page + seed), table_room=seed)


def test_page_map_again_gives_the_same():
    check_map(map_case(77, 8, 90, seed=3), repeat=3)
    check_map(map_case(5000, 8, 20, seed=4), repeat=3)


@pytest.mark.parametrize("requests", [40, 5001])
@pytest.mark.parametrize("short", [1, 10, 10 ** 9])
def test_page_map_when_the_pages_run_out(requests, short):
    for seed in range(3):
        want = check_map(map_case(requests, 4, 50, seed=seed, short=short, spare=0))
        assert want["unplaced"][0] > 0


def test_page_map_when_the_table_is_too_narrow():
    want = check_map(map_case(50, 4, 60, seed=8, width=9))
    assert want["unplaced"][0] > 0


@pytest.mark.parametrize("requests", [1, 100, 4500])
def test_page_map_without_new_tokens(requests):
    check_map(map_case(requests, 16, 100, seed=1, kind="nothing"))


def test_page_map_with_fewer_places_than_tokens():
    case = map_case(60, 8, 90, seed=12)
    check_map({**case, "tokens": case["tokens"] // 2})
    # a page whose first token has no place is not entered by that token: the step itself still has to enter it
    check_map({**case, "tokens": 0})


def test_page_map_of_no_requests():
    check_map(dict(page_size=4, lengths=np.zeros(0, np.int32), new_tokens=np.zeros(0, np.int32), pool=np.arange(6, dtype=np.int32),
                   cursor=np.array([1, 4], np.int64), table=np.zeros((0, 3), np.int32), tokens=5))


def test_page_map_takes_negative_lengths_for_none_and_skips_entries_that_are_no_pages():
    case = map_case(30, 8, 50, seed=21)
    case["lengths"][::7] = -3
    case["table"][1::5] = -1
    check_map(case)


def test_page_map_of_a_few_very_long_requests():
    case = dict(page_size=1 << 20, lengths=np.array([2 ** 31 - 5, 0, 5], np.int32), new_tokens=np.array([4, 1, -5], np.int32),
                pool=np.arange(3000, dtype=np.int32), cursor=np.array([2 ** 40, 2 ** 40 + 7], np.int64), table=np.full((3, 2100), 1 << 12, np.int32), tokens=9)
    check_map(case)


def test_page_map_of_more_tokens_than_can_be_counted():
    # four requests ask for 2^31-1 tokens each; few of them have an entry, and all pages there are get entered
    case = dict(page_size=1 << 22, lengths=np.array([7, 0, 1 << 22, 3], np.int32), new_tokens=np.array([2 ** 31 - 1 - 7, 2 ** 31 - 1, 2 ** 31 - 1 - (1 << 22), 2 ** 31 - 4], np.int32),
                pool=np.arange(1500, dtype=np.int32), cursor=np.array([3, 1400], np.int64), table=np.full((4, 600), -1, np.int32), tokens=33)
    case["table"][[0, 2, 3], 0] = [1450, 1451, 1452]
    want = check_map_counted(case)
    assert (want["table"] >= 0).sum() == 3 + 1397


# --------------------------------------------------------------------------- norm and rotation
def heads_case(tokens, hq, hk, dim, rotary, dtype, seed, axes=1, far=500, bad=False):
    import torch
    rng = np.random.default_rng(seed)
    # one projection's output, so that queries, keys and values are strided views
    qkv = gpu(rng.standard_normal((tokens, (hq + 2 * hk) * dim)).astype(np.float32), dtype)
    s = {"q": qkv[:, :hq * dim].view(tokens, hq, dim), "k": qkv[:, hq * dim:(hq + hk) * dim].view(tokens, hk, dim),
         "v": qkv[:, (hq + hk) * dim:].view(tokens, hk, dim), "q_weight": gpu(rng.uniform(0.5, 1.5, dim).astype(np.float32), dtype),
         "k_weight": gpu(rng.uniform(-1.5, 1.5, dim).astype(np.float32), dtype)}
    s["cos_sin"] = s["positions"] = s["axis_of"] = None
    if rotary:
        angle = rng.uniform(-np.pi, np.pi, (far, rotary // 2))
        s["cos_sin"] = gpu(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32))
        positions = rng.integers(0, far, (axes, tokens)).astype(np.int32)
        if bad and tokens:
            positions[0, ::3] = rng.choice([-1, far, 2 ** 31 - 1], positions[0, ::3].size)
        s["positions"] = gpu(positions)
        if axes > 1:
            axis_of = (np.arange(rotary // 2) % axes).astype(np.int32)
            if bad:
                axis_of[-1] = axes
            s["axis_of"] = gpu(axis_of)
    torch.cuda.synchronize()
    return s


def heads_want(s, eps, interleaved, which, weight=True):
    """The result in 64 bits and the magnitudes that bound its error."""
    x = host(s[which])
    w = host(s[which + "_weight"]) if weight else None
    c = d = None
    if s["cos_sin"] is not None:
        c, d = O.angles(host(s["cos_sin"]), host(s["positions"]), None if s["axis_of"] is None else host(s["axis_of"]))
    want = O.head_norm_rope(x, w, eps, c, d, interleaved)
    size = np.abs(O.head_norm_rope(x, w, eps, None, None, False))
    if c is not None:
        size = O.turned(size, np.ones_like(c), -np.ones_like(c), interleaved)          # |a| + |b| at a
        a, b = O._pairs(c.shape[1], interleaved)
        size[..., b] = size[..., a]
    return want, size


def check_heads(s, dtype, eps=1e-5, interleaved=False, weight=True, slots=None, page=16, pages=0, in_place=False, heads_first=False):
    import torch
    import paper_2407_13585_amd as fc
    want = {n: heads_want(s, eps, interleaved, n, weight) for n in "qk"}
    kw = {n: s[n] for n in ("q", "k", "cos_sin", "positions", "axis_of")}
    if weight:
        kw |= {n: s[n] for n in ("q_weight", "k_weight")}
    q_out = s["q"] if in_place else torch.full_like(s["q"], 7.0, memory_format=torch.contiguous_format)
    if slots is None:
        k_out = s["k"] if in_place else torch.full_like(s["k"], 7.0, memory_format=torch.contiguous_format)
        run([fc.HeadNormRope(q_out=q_out, k_out=k_out, eps=eps, interleaved=interleaved, **kw)])
        outs = {"q": q_out, "k": k_out}
    else:
        hk, dim = s["k"].shape[1:]
        shape = (pages, hk, page, dim) if heads_first else (pages, page, hk, dim)
        gen = torch.Generator("cuda").manual_seed(1)
        caches = [torch.randn(shape, device="cuda", generator=gen).to(types()[dtype]) for _ in range(2)]
        views = [c.transpose(1, 2) if heads_first else c for c in caches]
        before = [host(c) for c in views]
        run([fc.HeadNormRope(q_out=q_out, v=s["v"], k_cache=views[0], v_cache=views[1], slots=gpu(slots), eps=eps, interleaved=interleaved, **kw)])
        outs = {"q": q_out}
        at = np.asarray(slots)
        fine = (at >= 0) & (at < pages * page)
        tol = O.stored(np.zeros_like(before[0]), at, 20 * 2.0 ** -24 * want["k"][1] + U[dtype] * np.abs(want["k"][0]) + TINY[dtype])
        near(host(views[0]), O.stored(before[0], at, want["k"][0]), tol, "k_cache")
        assert np.array_equal(host(views[1]), O.stored(before[1], at, host(s["v"]))), "v_cache"
        assert fine.any() or not len(at) or np.array_equal(host(views[0]), before[0])
    for n, t in outs.items():
        ref, size = want[n]
        near(host(t), ref, 20 * 2.0 ** -24 * size + U[dtype] * np.abs(ref) + TINY[dtype], n)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim,rotary", [(2, 2), (8, 8), (32, 16), (64, 64), (72, 72), (80, 20), (96, 24), (100, 50), (126, 126), (128, 128), (128, 0),
                                        (192, 48), (256, 256), (512, 512)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_and_rotation_of_heads_of_any_size(dtype, dim, rotary, interleaved):
    if dim > 128 and rotary and rotary // 2 % 2:
        pytest.skip("refused")
    check_heads(heads_case(13, 5, 2, dim, rotary, dtype, seed=dim + rotary), dtype, interleaved=interleaved)


@pytest.mark.parametrize("tokens,hq,hk", [(0, 4, 2), (1, 1, 1), (1, 64, 8), (3, 7, 3), (17, 40, 0), (17, 0, 5), (255, 3, 1), (5001, 2, 1)])
def test_norm_and_rotation_of_few_and_many_tokens_and_heads(tokens, hq, hk):
    check_heads(heads_case(tokens, hq, hk, 64, 64, "bf16", seed=tokens), "bf16")
    check_heads(heads_case(tokens, hq, hk, 64, 32, "f32", seed=tokens), "f32", interleaved=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("axes", [1, 3])
def test_rotation_without_a_norm_and_positions_out_of_range(dtype, axes):
    check_heads(heads_case(31, 4, 2, 64, 64, dtype, seed=9, axes=axes), dtype, weight=False)
    check_heads(heads_case(31, 4, 2, 64, 48, dtype, seed=9, axes=axes, bad=True), dtype)
    check_heads(heads_case(31, 4, 2, 64, 48, dtype, seed=9, axes=axes, bad=True), dtype, interleaved=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("axes", [1, 3])
@pytest.mark.parametrize("dim,rotary", [(72, 18), (80, 20), (112, 28), (128, 128), (256, 250), (512, 46)])
def test_rotation_that_ends_inside_what_is_read_at_once(dtype, axes, dim, rotary):
    s = heads_case(29, 5, 2, dim, rotary, dtype, seed=dim + axes, axes=axes)
    check_heads(s, dtype, interleaved=True)
    check_grad(s, dtype, interleaved=True)
    wide = gpu(np.zeros((500, rotary + 3), np.float32))                                    # rows of angles that are not aligned
    wide[:, 1:1 + rotary] = s["cos_sin"]
    s["cos_sin"] = wide[:, 1:1 + rotary]
    check_heads(s, dtype, interleaved=True)
    if dim <= 128:
        check_heads(s, dtype)
        check_grad(s, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("axes", [1, 3])
def test_halves_that_do_not_lie_a_whole_read_apart(dtype, axes):
    for dim, rotary in [(72, 18), (80, 20), (112, 28), (72, 36)]:
        slots = np.random.default_rng(dim).permutation(80)[:37].astype(np.int64)
        slots[::6] = -1
        check_heads(heads_case(37, 19, 6, dim, rotary, dtype, seed=dim, axes=axes), dtype, slots=slots, page=8, pages=10)
        check_heads(heads_case(37, 19, 6, dim, rotary, dtype, seed=dim, axes=axes, bad=True), dtype)
        check_heads(heads_case(300, 3, 2, dim, rotary, dtype, seed=dim, axes=axes), dtype, weight=False, in_place=True)
        check_grad(heads_case(700, 9, 2, dim, rotary, dtype, seed=dim, axes=axes), dtype)
        check_grad(heads_case(5, 40, 8, dim, rotary, dtype, seed=dim, axes=axes), dtype, weight=False, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
def test_norm_and_rotation_in_place(dtype):
    check_heads(heads_case(77, 6, 3, 96, 96, dtype, seed=2), dtype, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page,heads_first", [(1, False), (16, False), (24, True), (7, True)])
def test_keys_and_values_go_into_the_cache(dtype, page, heads_first):
    pages = 90 // page + 3
    for tokens in (1, 8, 61):
        slots = np.random.default_rng(tokens).permutation(pages * page)[:tokens].astype(np.int64)
        slots[::5] = [-1, pages * page, -2 ** 40, 2 ** 33][tokens % 4]
        check_heads(heads_case(tokens, 6, 3, 64, 64, dtype, seed=tokens), dtype, slots=slots, page=page, pages=pages, heads_first=heads_first)


def test_norm_of_zeros_and_of_values_that_are_not_finite():
    s = heads_case(9, 3, 2, 64, 32, "f32", seed=4)
    s["q"][0] = 0.0
    s["q"][1, 1, 5] = math.inf
    s["q"][2, 0, 7] = math.nan
    s["k"][3, 1] = 1e-30
    import torch
    import paper_2407_13585_amd as fc
    out = [torch.empty((9, h, 64), device="cuda") for h in (3, 2)]
    run([fc.HeadNormRope(q=s["q"], k=s["k"], q_out=out[0], k_out=out[1], q_weight=s["q_weight"], k_weight=s["k_weight"], cos_sin=s["cos_sin"],
                         positions=s["positions"])])
    q, k = (host(t) for t in out)
    assert (q[0] == 0).all() and np.isnan(q[2, 0]).all() and np.isnan(q[1, 1]).any() and np.isfinite(q[3:]).all() and np.isfinite(q[1, 0]).all()
    near(k, heads_want(s, 1e-6, False, "k")[0], 20 * 2.0 ** -24 * heads_want(s, 1e-6, False, "k")[1] + 1e-37)


def check_grad(s, dtype, eps=1e-5, interleaved=False, weight=True, in_place=False, seed=0):
    import torch
    import paper_2407_13585_amd as fc
    rng = np.random.default_rng(seed)
    dy = {n: gpu(rng.standard_normal(tuple(s[n].shape)).astype(np.float32), dtype) for n in "qk"}
    c = d = None
    if s["cos_sin"] is not None:
        c, d = O.angles(host(s["cos_sin"]), host(s["positions"]), None if s["axis_of"] is None else host(s["axis_of"]))
    want = {}
    for n in "qk":
        x, g, w = host(s[n]), host(dy[n]), host(s[n + "_weight"]) if weight else None
        dx, dw = O.head_norm_rope_grad(x, w, eps, c, d, interleaved, g)
        size = np.abs(g)
        if c is not None:
            size = O.turned(size, np.ones_like(c), -np.ones_like(c), interleaved)
            a, b = O._pairs(c.shape[1], interleaved)
            size[..., b] = size[..., a]
        terms = 0.0
        if weight:
            r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
            terms = (size * np.abs(x * r)).sum((0, 1))
            size = r * (np.abs(w) * size + np.abs(x * r) * (np.abs(w) * size * np.abs(x * r)).mean(-1, keepdims=True))
        want[n] = dx, dw, size, terms
    dx = dy if in_place else {n: torch.full_like(dy[n], 7.0) for n in "qk"}
    kw = {n: s[n] for n in ("q", "k", "cos_sin", "positions", "axis_of")}
    dw = {}
    if weight:
        dw = {n: torch.full((s["q"].shape[2],), 7.0, device="cuda") for n in "qk"}
        kw |= {"q_weight": s["q_weight"], "k_weight": s["k_weight"], "dq_weight": dw["q"], "dk_weight": dw["k"]}
    run([fc.HeadNormRopeGrad(dq_out=dy["q"], dk_out=dy["k"], dq=dx["q"], dk=dx["k"], eps=eps, interleaved=interleaved, **kw)], repeat=1 if in_place else 2)
    for n in "qk":
        ref, refw, size, terms = want[n]
        near(host(dx[n]), ref, 48 * 2.0 ** -24 * size + U[dtype] * np.abs(ref) + TINY[dtype], "d" + n)
        if weight:
            near(host(dw[n]), refw, 1e-5 * terms + 1e-37, f"d{n}_weight")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim,rotary", [(2, 2), (64, 64), (72, 72), (80, 20), (96, 24), (126, 126), (128, 128), (128, 0), (256, 256), (512, 512)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_for_heads_of_any_size(dtype, dim, rotary, interleaved):
    check_grad(heads_case(13, 5, 2, dim, rotary, dtype, seed=dim + rotary), dtype, interleaved=interleaved)


@pytest.mark.parametrize("tokens,hq,hk", [(0, 4, 2), (1, 1, 1), (1, 64, 8), (3, 7, 3), (17, 40, 0), (17, 0, 5), (255, 3, 1), (5001, 2, 1)])
def test_gradient_of_few_and_many_tokens_and_heads(tokens, hq, hk):
    check_grad(heads_case(tokens, hq, hk, 64, 64, "bf16", seed=tokens), "bf16")
    check_grad(heads_case(tokens, hq, hk, 64, 32, "f32", seed=tokens, axes=3), "f32", interleaved=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_without_a_norm_and_in_place(dtype):
    check_grad(heads_case(31, 4, 2, 64, 64, dtype, seed=9), dtype, weight=False)
    check_grad(heads_case(77, 6, 3, 96, 48, dtype, seed=2), dtype, in_place=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hk", [(3, 1), (9, 2)])
def test_norm_and_gradient_with_an_eps_of_zero(dtype, hq, hk):
    # rows of a wave that no head has are zeros, whose norm is not finite without eps: nothing of them may reach the weights' gradients
    s = heads_case(11, hq, hk, 64, 64, dtype, seed=hq)
    check_heads(s, dtype, eps=0.0)
    check_grad(s, dtype, eps=0.0)


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_against_differences(interleaved):
    # along a random direction, central differences of the definition: their own error is of second order in the step
    import torch
    import paper_2407_13585_amd as fc
    s = heads_case(6, 3, 2, 64, 48, "f32", seed=31)
    rng = np.random.default_rng(1)
    c, d = O.angles(host(s["cos_sin"]), host(s["positions"]), None)
    dy = {n: rng.standard_normal(tuple(s[n].shape)).astype(np.float32) for n in "qk"}
    out = {n: torch.empty(tuple(s[n].shape), device="cuda") for n in "qk"}
    dw = {n: torch.empty(64, device="cuda") for n in "qk"}
    run([fc.HeadNormRopeGrad(q=s["q"], k=s["k"], dq_out=gpu(dy["q"]), dk_out=gpu(dy["k"]), dq=out["q"], dk=out["k"], dq_weight=dw["q"],
                             dk_weight=dw["k"], q_weight=s["q_weight"], k_weight=s["k_weight"], cos_sin=s["cos_sin"], positions=s["positions"],
                             interleaved=interleaved)])
    h = 1e-5
    for n in "qk":
        x, w = host(s[n]), host(s[n + "_weight"])
        value = lambda x, w: float((O.head_norm_rope(x, w, 1e-6, c, d, interleaved) * dy[n]).sum())  # noqa: E731
        for along_x in (True, False):
            v = rng.standard_normal(x.shape if along_x else w.shape)
            slope = (value(x + h * v, w) - value(x - h * v, w) if along_x else value(x, w + h * v) - value(x, w - h * v)) / (2 * h)
            got = float((host(out[n] if along_x else dw[n]) * v).sum())
            scale = float(np.abs(host(out[n] if along_x else dw[n]) * v).sum())
            assert abs(got - slope) <= 1e-5 * scale, (n, along_x, got, slope)


def test_weight_gradients_are_the_same_bits_every_time():
    import torch
    import paper_2407_13585_amd as fc
    s = heads_case(4001, 5, 3, 64, 64, "bf16", seed=8)
    dy = {n: torch.randn(s[n].shape, device="cuda").to(torch.bfloat16) for n in "qk"}
    seen = []
    for _ in range(3):
        dw = [torch.empty(64, device="cuda") for _ in "qk"]
        run([fc.HeadNormRopeGrad(q=s["q"], k=s["k"], dq_out=dy["q"], dk_out=dy["k"], dq=torch.empty_like(dy["q"]), dk=torch.empty_like(dy["k"]),
                                 dq_weight=dw[0], dk_weight=dw[1], q_weight=s["q_weight"], k_weight=s["k_weight"], cos_sin=s["cos_sin"],
                                 positions=s["positions"])])
        seen.append([host(t) for t in dw])
    assert all(np.array_equal(a, b) for again in seen[1:] for a, b in zip(seen[0], again))


# --------------------------------------------------------------------------- attention
def attention_case(lengths, hq, hk, dim, page, dtype, seed, heads_first=False, spare_width=1, poison=True, sharp=1.0):
    """Pages in random order; what lies past the lengths, in the cache and in the table, is not a number / not a page."""
    import torch
    rng = np.random.default_rng(seed)
    lengths = np.asarray(lengths, np.int32)
    have = -(-np.maximum(lengths, 0) // page)
    width = int(have.max(initial=0)) + spare_width
    pages = int(have.sum()) + 2
    order = rng.permutation(pages)[:int(have.sum())]
    table = rng.choice([-1, pages, 2 ** 31 - 1, -2 ** 31], (len(lengths), width)).astype(np.int32)
    table[np.arange(width)[None, :] < have[:, None]] = order
    k, v = (rng.standard_normal((pages, page, hk, dim)).astype(np.float32) for _ in range(2))
    if poison:
        used = np.zeros((pages, page), bool)
        for b, n in enumerate(lengths):
            for j in range(max(int(n), 0)):
                used[table[b, j // page], j % page] = True
        k[~used] = np.resize([math.nan, math.inf, -math.inf], k[~used].shape)
        v[~used] = np.resize([math.inf, math.nan], v[~used].shape)
    caches = []
    for c in (k, v):
        t = gpu(c, dtype)
        caches.append(t.transpose(1, 2).contiguous().transpose(1, 2) if heads_first else t)
    q = gpu((sharp * rng.standard_normal((len(lengths), hq, dim))).astype(np.float32), dtype)
    torch.cuda.synchronize()
    return {"q": q, "k_cache": caches[0], "v_cache": caches[1], "table": gpu(table), "lengths": gpu(lengths)}


def attention_want(s, scale, window):
    k, v = host(s["k_cache"]), host(s["v_cache"])
    return O.paged_attention(host(s["q"]), k, v, host(s["table"]), host(s["lengths"]), scale, window)


def check_attention(s, dtype, window=0, scale=None, lse=True, want=None, stream=None):
    import torch
    import paper_2407_13585_amd as fc
    batch, hq, dim = s["q"].shape
    scale = dim ** -0.5 if scale is None else scale
    out = torch.full((batch, hq, dim), 7.0, dtype=s["q"].dtype, device="cuda")
    logs = torch.full((batch, hq), 7.0, device="cuda") if lse else None
    if stream is not None:
        torch.cuda.synchronize()
    run([fc.PagedAttention(out=out, lse=logs, scale=scale, window=window, **s)], stream=stream)
    ref, ref_lse, reach, spread = want or attention_want(s, scale, window)
    e = (dim + 8) * 2.0 ** -24 * reach
    near(host(out), ref, 2 * (e[..., None] + 2.0 ** -20 + 2.0 ** -16) * spread + U[dtype] * np.abs(ref) + TINY[dtype], "out")
    if lse:
        near(host(logs), ref_lse, e + 2.0 ** -20 * (1 + np.abs(np.where(np.isfinite(ref_lse), ref_lse, 0))), "lse")
    return host(out), host(logs) if lse else None


LENGTHS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 257, 511, 700]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page", [1, 3, 8, 16, 24, 32, 48, 64, 100])
def test_attention_over_pages_of_any_size_and_lengths_around_every_tile(dtype, page):
    check_attention(attention_case(LENGTHS, 4, 2, 64, page, dtype, seed=page, heads_first=page % 2 == 0), dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim", [8, 16, 40, 64, 72, 80, 96, 112, 128, 136, 192, 200, 256])
def test_attention_for_heads_of_any_size(dtype, dim):
    check_attention(attention_case([0, 1, 40, 77, 130], 6, 3, dim, 16, dtype, seed=dim), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hk", [(1, 1), (5, 5), (7, 1), (16, 1), (17, 1), (24, 1), (64, 2), (66, 2), (48, 8)])
def test_attention_with_groups_of_any_size(dtype, hq, hk):
    check_attention(attention_case([3, 0, 97, 33], hq, hk, 64, 16, dtype, seed=hq), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [1, 2, 16, 31, 100, 10 ** 6])
def test_attention_in_a_window(dtype, window):
    s = attention_case(LENGTHS, 4, 2, 64, 16, dtype, seed=window)
    check_attention(s, dtype, window=window)
    check_attention(attention_case(LENGTHS, 4, 2, 64, 7, dtype, seed=window), dtype, window=window)


@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 64), ("f32", 128)])
def test_attention_split_over_a_long_cache(dtype, dim):
    for lengths in ([5000], [4097, 0, 1, 3000], [1] * 40 + [6000]):
        check_attention(attention_case(lengths, 8, 2, dim, 16, dtype, seed=len(lengths), poison=len(lengths) < 40), dtype)


def test_attention_of_no_requests_and_negative_lengths():
    check_attention(attention_case(np.zeros(0, np.int32), 4, 2, 64, 16, "bf16", seed=1), "bf16")
    check_attention(attention_case([-5, 3, -2 ** 31], 4, 2, 64, 16, "bf16", seed=1), "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_skips_pages_outside_the_cache_and_the_table(dtype):
    s = attention_case([100, 64, 200, 40], 4, 2, 64, 16, dtype, seed=5)
    table = host(s["table"]).copy()
    table[0, 2], table[1, :], table[2, 11] = -1, 2 ** 31 - 1, s["k_cache"].shape[0]
    s["table"] = gpu(table)
    check_attention(s, dtype)
    s["lengths"] = gpu(np.array([10 ** 9, 2 ** 31 - 1, 500, 40], np.int32))              # beyond the table
    s["k_cache"], s["v_cache"] = (c.nan_to_num(0.5, 0.25, -0.25) for c in (s["k_cache"], s["v_cache"]))
    check_attention(s, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_attention_with_large_scores(dtype):
    s = attention_case([1, 50, 300], 4, 2, 64, 16, dtype, seed=11, sharp=40.0)
    check_attention(s, dtype)
    check_attention(s, dtype, scale=-3.0)
    check_attention(s, dtype, scale=0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_values_that_are_not_finite(dtype):
    # a NaN among a request's keys makes its heads NaN; an infinite value of a key with a weight is an infinite sum; the others stay
    s = attention_case([90, 90, 90, 90], 2, 2, 64, 16, dtype, seed=3)
    k, v = s["k_cache"], s["v_cache"]
    table = host(s["table"])
    k[int(table[0, 1]), 3, 0, 5] = math.nan
    v[int(table[1, 2]), 7, 1, 9] = math.inf
    v[int(table[2, 0]), 0, 0, 2] = -math.inf
    out, lse = (host(x) for x in attention_raw(s))
    ref, ref_lse, _, _ = attention_want(s, 0.125, 0)
    assert np.isnan(out[0, 0]).all() and np.isnan(lse[0, 0])
    assert out[1, 1, 9] == math.inf and np.isfinite(np.delete(out[1, 1], 9)).all()
    assert out[2, 0, 2] == -math.inf and np.isfinite(np.delete(out[2, 0], 2)).all()
    for b, h in ((0, 1), (1, 0), (2, 1), (3, 0), (3, 1)):
        near(out[b, h], ref[b, h], 2 ** -7 if dtype == "bf16" else 1e-4)
        near(lse[b, h:h + 1], ref_lse[b, h:h + 1], 1e-4)


def attention_raw(s, **kw):
    import torch
    import paper_2407_13585_amd as fc
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], device="cuda")
    run([fc.PagedAttention(out=out, lse=lse, **s, **kw)])
    return out, lse


def test_attention_on_strided_tensors_and_without_lse():
    import torch
    import paper_2407_13585_amd as fc
    s = attention_case([5, 70, 129], 6, 2, 64, 16, "bf16", seed=6)
    want = attention_want(s, 0.125, 0)
    wide = torch.zeros((3, 6, 3, 64), dtype=torch.bfloat16, device="cuda")
    wide[:, :, 1] = s["q"]
    out = torch.full((6, 3, 80), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((6, 3 * 2), 9.0, device="cuda").t()[::2].contiguous()
    table = torch.full((3, 40), -5, dtype=torch.int32, device="cuda")
    table[:, 1:1 + s["table"].shape[1]] = s["table"]
    view = out[:, :, 8:72].transpose(0, 1)
    run([fc.PagedAttention(q=wide[:, :, 1], k_cache=s["k_cache"], v_cache=s["v_cache"], table=table[:, 1:1 + s["table"].shape[1]],
                           lengths=s["lengths"], out=view, lse=lse)])
    near(host(view), want[0], 2.0 ** -8 * np.abs(want[0]) + 2.0 ** -14 * (1 + want[3]))
    near(host(lse), want[1], 1e-5 * (1 + np.abs(want[1])))
    assert (out[:, :, :8] == 9).all() and (out[:, :, 72:] == 9).all()
    check_attention(s, "bf16", lse=False)
    same = {**s, "q": s["q"][:1].expand(3, 6, 64)}                                        # one query for all requests: stride 0
    check_attention(same, "bf16")


@pytest.mark.parametrize("dim,page", [(64, 16), (192, 48), (256, 5)])
def test_attention_of_32_bits_keeps_its_precision(dim, page):
    """Root mean square of the error, relative to that of the result.

    A score of n = dim products, its own size 2 here, is off by 2 * 2^-24 sqrt(n / 6) where they are summed one by one (7.8e-7 for 256), and by half of
    it in four sums; weights are off by as much of themselves, and the output, a sum of values of either sign, by as much of its size.
    With 2^-23 for the powers, their sum and the quotient: 5.1e-7 at most for 256."""
    s = attention_case([1728, 900, 333], 20, 5, dim, page, "f32", seed=dim, sharp=2.0)
    out, lse = check_attention(s, "f32")
    ref, ref_lse = attention_want(s, dim ** -0.5, 0)[:2]
    rms = lambda x: np.sqrt(np.mean(np.square(x)))  # noqa: E731
    assert rms(out - ref) <= (2.0 ** -24 * math.sqrt(dim / 6) + 2.0 ** -23) * rms(ref)
    assert rms(lse - ref_lse) <= 2.0 ** -24 * rms(ref_lse)


def many_short(dtype, seed, requests=300, longest=None):
    """More rows than workgroups are resident, none longer than two steps of a workgroup, unless `longest` says so."""
    rng = np.random.default_rng(seed)
    lengths = rng.integers(0, 129 if dtype == "f32" else 257, requests)
    lengths[:len(LENGTHS)] = np.minimum(LENGTHS, 128 if dtype == "f32" else 256)
    if longest:
        lengths[requests // 2] = longest
    return lengths


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim,page,heads_first", [(64, 16, False), (40, 24, True), (128, 16, True), (128, 5, False), (96, 32, False), (192, 48, False), (256, 7, True)])
def test_attention_of_many_short_rows(dtype, dim, page, heads_first):
    s = attention_case(many_short(dtype, dim + page), 8, 4, dim, page, dtype, seed=dim, heads_first=heads_first)
    check_attention(s, dtype)
    if dim in (64, 128):
        check_attention(s, dtype, window=37)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hk", [(4, 4), (17, 1), (66, 2)])
def test_attention_of_many_short_rows_with_groups_of_any_size(dtype, hq, hk):
    check_attention(attention_case(many_short(dtype, hq, requests=1200 // (hk * -(-hq // hk // 16))), hq, hk, 64, 16, dtype, seed=hq), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_many_short_rows_and_one_that_is_not(dtype):
    check_attention(attention_case(many_short(dtype, 1, longest=1500), 8, 4, 64, 16, dtype, seed=21), dtype)


def test_attention_of_many_short_rows_into_rows_that_are_not_aligned_and_over_missing_pages():
    import torch
    import paper_2407_13585_amd as fc
    s = attention_case(many_short("bf16", 2), 8, 4, 64, 16, "bf16", seed=22)
    holes = torch.rand(s["table"].shape, generator=torch.Generator().manual_seed(23)).cuda() < 0.3
    s["table"][holes] = -1
    want = attention_want(s, 0.125, 0)
    out = torch.full((300, 8, 65), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty((300, 8), device="cuda")
    run([fc.PagedAttention(out=out[:, :, 1:], lse=lse, **s)])
    near(host(out[:, :, 1:]), want[0], 2.0 ** -8 * np.abs(want[0]) + 2.0 ** -14 * (1 + want[3]))
    near(host(lse), want[1], 1e-5 * (1 + np.abs(want[1])))
    assert (out[:, :, 0] == 9).all()


def test_attention_gives_the_same_bits_every_time():
    s = attention_case([3000, 1, 777], 8, 2, 128, 16, "bf16", seed=14, poison=False)
    first = [host(t) for t in attention_raw(s)]
    for _ in range(3):
        assert all(np.array_equal(a, host(b)) for a, b in zip(first, attention_raw(s)))


@pytest.mark.parametrize("heads_first", [False, True])
def test_attention_and_append_beyond_32_bit_offsets(heads_first):
    # a cache of more than 2^32 elements: the pages in use lie at its far end
    import torch
    import paper_2407_13585_amd as fc
    pages, page, hk, dim = (1 << 32) // (16 * 2 * 64) + 9, 16, 2, 64
    shape = (pages, hk, page, dim) if heads_first else (pages, page, hk, dim)
    caches = [torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    views = [c.transpose(1, 2) if heads_first else c for c in caches]
    far = np.array([pages - 1, pages - 5, pages - 3], np.int32)
    gen = torch.Generator("cuda").manual_seed(2)
    for c in caches:
        c[-9:] = torch.randn(c[-9:].shape, device="cuda", generator=gen).to(torch.bfloat16)
    s = heads_case(1, 4, 2, 64, 64, "bf16", seed=1)
    slot = int(far[1]) * page + 3
    q_out = torch.empty((1, 4, 64), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.empty_like(q_out), torch.empty((1, 4), device="cuda")
    run([fc.HeadNormRope(q=s["q"], k=s["k"], v=s["v"], q_out=q_out, k_cache=views[0], v_cache=views[1], slots=gpu(np.array([slot])),
                         q_weight=s["q_weight"], k_weight=s["k_weight"], cos_sin=s["cos_sin"], positions=s["positions"]),
         fc.PagedAttention(q=q_out, k_cache=views[0], v_cache=views[1], table=gpu(far[None, :]), lengths=gpu(np.array([20], np.int32)), out=out, lse=lse)])
    small = [host(v[-9:]) for v in views]
    near(small[0][-5, 3][None], heads_want(s, 1e-6, False, "k")[0], 2.0 ** -7)
    assert np.array_equal(small[1][-5, 3][None], host(s["v"]))
    ref, ref_lse, _, spread = O.paged_attention(host(q_out), small[0], small[1], (far - (pages - 9))[None, :], [20], 0.125)
    near(host(out), ref, 2.0 ** -8 * np.abs(ref) + 2.0 ** -14 * (1 + spread))
    near(host(lse), ref_lse, 1e-5 * (1 + np.abs(ref_lse)))
    del caches, views
    torch.cuda.empty_cache()


# --------------------------------------------------------------------------- together
def test_operators_run_on_the_stream_they_are_given():
    import torch
    side = torch.cuda.Stream()
    s = attention_case([100, 40], 4, 2, 64, 16, "bf16", seed=2)
    check_attention(s, "bf16", stream=side)


def test_a_list_of_operators_replays_from_a_graph_and_matches_the_eager_step():
    # a decoding step: new slots and pages, heads into the cache, attention over what is then there
    import torch
    import paper_2407_13585_amd as fc
    batch, hq, hk, dim, page, width, pages = 5, 4, 2, 64, 8, 12, 64
    rng = np.random.default_rng(4)
    lengths = np.array([0, 7, 8, 30, 17], np.int32)
    have = -(-lengths // page)
    order = rng.permutation(pages).astype(np.int32)
    table = np.full((batch, width), -1, np.int32)
    table[np.arange(width)[None, :] < have[:, None]] = order[:have.sum()]
    free = order[have.sum():]
    pool = np.concatenate([free, np.zeros(pages - free.size, np.int32)]).astype(np.int32)
    angle = rng.uniform(-3, 3, (200, dim // 2))
    t = {"lengths": gpu(lengths), "new": gpu(np.ones(batch, np.int32)), "pool": gpu(pool), "cursor": gpu(np.array([0, free.size], np.int64)), "table": gpu(table),
         "after": gpu(np.zeros(batch, np.int32)), "row": gpu(np.zeros(batch + 1, np.int32)), "slots": gpu(np.zeros(batch, np.int64)),
         "positions": gpu(np.zeros(batch, np.int32)), "request": gpu(np.zeros(batch, np.int32)), "cursor_after": gpu(np.zeros(2, np.int64)),
         "unplaced": gpu(np.zeros(1, np.int64)), "cos_sin": gpu(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)),
         "q": gpu(np.zeros((batch, hq, dim), np.float32), "bf16"), "k": gpu(np.zeros((batch, hk, dim), np.float32), "bf16"),
         "v": gpu(np.zeros((batch, hk, dim), np.float32), "bf16"), "w": gpu(np.ones(dim, np.float32), "bf16")}
    t["q_out"], t["out"] = torch.empty_like(t["q"]), torch.empty_like(t["q"])
    caches = [torch.zeros((pages, page, hk, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    ops = [fc.PageMap(page_size=page, lengths=t["lengths"], new_tokens=t["new"], pool=t["pool"], cursor=t["cursor"], table=t["table"],
                      lengths_after=t["after"], row_start=t["row"], slots=t["slots"], positions=t["positions"], request=t["request"],
                      cursor_after=t["cursor_after"], unplaced=t["unplaced"]),
           fc.HeadNormRope(q=t["q"], k=t["k"], v=t["v"], q_out=t["q_out"], k_cache=caches[0], v_cache=caches[1], slots=t["slots"], q_weight=t["w"],
                           k_weight=t["w"], cos_sin=t["cos_sin"], positions=t["positions"].view(1, -1)),
           fc.PagedAttention(q=t["q_out"], k_cache=caches[0], v_cache=caches[1], table=t["table"], lengths=t["after"], out=t["out"])]
    scratch = torch.zeros(fc.fc_operators_scratch_bytes(ops), dtype=torch.uint8, device="cuda")
    bound = fc.BoundOperators(ops, scratch)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        bound(side.cuda_stream)                              # the first call, outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        bound(torch.cuda.current_stream().cuda_stream)
    names = ("after", "row", "slots", "positions", "request", "cursor_after", "unplaced", "q_out", "out", "table", "pool")
    for step in range(4):
        for n in "qkv":
            t[n].copy_(gpu(rng.standard_normal(tuple(t[n].shape)).astype(np.float32), "bf16"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = {n: host(t[n]) for n in names}
        for n in ("q_out", "out", "slots"):
            t[n].fill_(3)
        fc.fc_run_operators(ops, scratch, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert all(np.array_equal(got[n], host(t[n])) for n in names), step
        ref, _, _, spread = O.paged_attention(got["q_out"], host(caches[0]), host(caches[1]), got["table"], got["after"], dim ** -0.5)
        near(got["out"], ref, 2.0 ** -8 * np.abs(ref) + 2.0 ** -14 * (1 + spread))
        assert got["unplaced"][0] == 0 and (got["after"] == host(t["lengths"]) + 1).all()
        t["lengths"].copy_(t["after"])
        t["cursor"].copy_(t["cursor_after"])
        fc.fc_check(scratch)
