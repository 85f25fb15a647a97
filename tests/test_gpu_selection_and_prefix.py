"""Bounds of pages, the selection of pages by them, attention over the selected pages and over shared prefixes, on the GPU against the
definitions in 64 bits (oracle/cache.py).

Bounds are keys, so they are equal; scores of 64 bits differ by 2^-53 of the terms' magnitudes at most whatever their order, which no two scores
of these inputs come near, so selections are equal.  Tolerances of attention: those of one table a request (test_gpu_operators.py), whose rounding
is the same: (D + 8) 2^-24 of the magnitudes for a score, 2^-20 for a weight, 2^-16 for what a weight is held in, half a step of the result."""
import math

import numpy as np
import pytest

from oracle import cache as O
from test_gpu_operators import TINY, U, gpu, host, near, run

pytestmark = pytest.mark.gpu

POISON = [math.nan, math.inf, -math.inf]
NO_PAGE = [-1, 2 ** 31 - 1, -2 ** 31]


def caches_of(rng, pages, page, hk, dim, dtype, used, heads_first, count=2):
    """`count` caches whose places outside `used` [pages, page] hold what is not finite."""
    found = []
    for _ in range(count):
        c = rng.standard_normal((pages, page, hk, dim)).astype(np.float32)
        c[~used] = np.resize(POISON, c[~used].shape)
        t = gpu(c, dtype)
        found.append(t.transpose(1, 2).contiguous().transpose(1, 2) if heads_first else t)
    return found


def pages_for(rng, page, *lists, spare=2, width=None):
    """A table in random order for each list of lengths, no page behind them; the pages there are, and which of their places are in use."""
    have = [-(-np.maximum(n, 0) // page) for n in lists]
    total = sum(int(h.sum()) for h in have)
    pages = total + spare
    order, at, used, tables = rng.permutation(pages)[:total], 0, np.zeros((pages, page), bool), []
    for n, h in zip(lists, have):
        table = rng.choice(NO_PAGE + [pages], h.shape + ((width or int(h.max(initial=0))) + 1,)).astype(np.int32)
        for i in np.ndindex(h.shape):
            mine = order[at:at + h[i]]
            table[i][:h[i]] = mine
            at += h[i]
            used[mine] = True
            if n[i] > 0 and n[i] % page:
                used[mine[-1], n[i] % page:] = False
        tables.append(table)
    return tables, pages, used


def close(got, want, dtype, dim, what="out", lse=None, ref_lse=None):
    ref, logs, reach, spread = want
    e = (dim + 8) * 2.0 ** -24 * reach
    near(got, ref, 2 * (e[..., None] + 2.0 ** -20 + 2.0 ** -16) * spread + U[dtype] * np.abs(ref) + TINY[dtype], what)
    if lse is not None:
        near(lse, logs, e + 2.0 ** -20 * (1 + np.abs(np.where(np.isfinite(logs), logs, 0))), "lse")


# --------------------------------------------------------------------------- bounds of pages
STEPS = [(0, 0), (0, 1), (5, 6), (5, 5), (7, 3), (15, 16), (16, 17), (15, 17), (0, 100), (3, 64), (-4, 5), (-3, -1), (31, 200), (250, 257)]


def bounds_case(steps, hk, dim, page, dtype, seed, heads_first=False):
    rng = np.random.default_rng(seed)
    before, after = (np.array(x, np.int32) for x in zip(*steps))
    (table,), pages, used = pages_for(rng, page, np.maximum(after, before))
    k, = caches_of(rng, pages, page, hk, dim, dtype, used, heads_first, count=1)
    bounds = gpu(np.sort(rng.standard_normal((pages, hk, 2, dim)).astype(np.float32), axis=2), dtype)
    return {"k_cache": k, "table": gpu(table), "lengths_before": gpu(before), "lengths": gpu(after), "bounds": bounds}


def check_bounds(s, repeat=1):
    import paper_2407_13585_amd as fc
    want = O.page_bounds(*(host(s[n]) for n in ("k_cache", "table", "lengths_before", "lengths", "bounds")))
    run([fc.PageBounds(**s)], repeat=repeat)
    got = host(s["bounds"])
    assert np.array_equal(got, want, equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page", [1, 3, 16, 24, 100])
def test_bounds_of_pages_of_any_size(dtype, page):
    check_bounds(bounds_case(STEPS, 3, 64, page, dtype, seed=page, heads_first=page % 2 == 0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [8, 16, 40, 72, 96, 128, 200, 256])
def test_bounds_of_heads_of_any_size(dtype, dim):
    check_bounds(bounds_case(STEPS[:10], 2, dim, 16, dtype, seed=dim))


@pytest.mark.parametrize("requests", [1, 255, 256, 257, 2000])
def test_bounds_of_few_and_many_requests(requests):
    rng = np.random.default_rng(requests)
    before = rng.integers(0, 40, requests)
    steps = list(zip(before, before + rng.choice([0, 0, 1, 5, 30], requests)))
    check_bounds(bounds_case(steps, 2, 16, 8, "bf16", seed=requests))


def test_bounds_again_give_the_same():
    check_bounds(bounds_case(STEPS, 2, 64, 16, "bf16", seed=1), repeat=3)


def test_bounds_of_no_requests_and_of_lengths_beyond_the_table():
    check_bounds(bounds_case([(0, 0)], 2, 64, 16, "bf16", seed=1))
    s = bounds_case([(3, 40), (0, 16), (10, 90)], 2, 64, 16, "bf16", seed=2)
    s["lengths"] = gpu(np.array([2 ** 31 - 1, 16, 500], np.int32))
    s["table"] = s["table"][:, :2].contiguous()
    check_bounds(s)
    s["lengths_before"] = gpu(np.array([2 ** 31 - 2, 2 ** 31 - 1, 31], np.int32))
    check_bounds(s)


def test_bounds_leave_out_pages_that_are_not_there():
    s = bounds_case([(3, 40), (0, 100), (10, 90)], 2, 64, 16, "f16", seed=3)
    table = host(s["table"]).copy()
    table[0, 0], table[1, 2:5], table[2, 5] = -1, [2 ** 31 - 1, s["k_cache"].shape[0], -2 ** 31], -7
    s["table"] = gpu(table)
    check_bounds(s)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_bounds_of_keys_that_are_not_finite(dtype):
    s = bounds_case([(5, 20), (0, 64), (0, 30)], 2, 64, 16, dtype, seed=4)
    table, k = host(s["table"]), s["k_cache"]
    k[int(table[0, 0]), 7, 0, 3] = math.nan
    k[int(table[0, 1]), 0, 1, 63] = -math.inf
    k[int(table[1, 2]), 15, 1, 9] = math.inf
    s["bounds"][int(table[0, 0]), 1, 0, 40] = math.nan       # of the keys before
    s["bounds"][int(table[1, 0]), 1, 1, 2] = math.nan        # an earlier request's
    check_bounds(s)
    got = host(s["bounds"])
    assert np.isnan(got[table[0, 0], 0, :, 3]).all() and np.isnan(got[table[0, 0], 1, 0, 40]) and np.isfinite(got[table[1, 0], 1, 1, 2])


def test_bounds_in_a_strided_array_leave_what_lies_between():
    import torch
    s = bounds_case([(3, 40), (0, 16)], 3, 40, 16, "bf16", seed=5)
    wide = torch.full((s["bounds"].shape[0], 4, 3, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 1:, 1:, 8:48] = s["bounds"]
    s["bounds"] = wide[:, 1:, 1:, 8:48]
    check_bounds(s)
    assert (wide[:, 0] == 9).all() and (wide[:, :, 0] == 9).all() and (wide[..., :8] == 9).all() and (wide[..., 48:] == 9).all()


# --------------------------------------------------------------------------- selection
def select_case(lengths, hq, hk, dim, page, most, dtype, seed, width=None, bounds=None):
    import torch
    rng = np.random.default_rng(seed)
    lengths = np.asarray(lengths, np.int32)
    (table,), pages, used = pages_for(rng, page, lengths, width=width)
    if bounds is None:
        bounds = np.sort(rng.standard_normal((pages, hk, 2, dim)).astype(np.float32), axis=2) + rng.standard_normal((pages, hk, 1, 1)).astype(np.float32)
        bounds[~used.any(1)] = math.nan
    return {"q": gpu(rng.standard_normal((len(lengths), hq, dim)).astype(np.float32), dtype), "bounds": gpu(bounds, dtype), "table": gpu(table),
            "lengths": gpu(lengths), "selected": torch.full((len(lengths), hk, most), 77, dtype=torch.int32, device="cuda"),
            "selected_lengths": torch.full((len(lengths), hk), 77, dtype=torch.int32, device="cuda")}


def check_select(s, page, first=1, last=1):
    import paper_2407_13585_amd as fc
    run([fc.PageSelect(page_size=page, first=first, last=last, **s)])
    want, held = O.page_select(*(host(s[n]) for n in ("q", "bounds", "table", "lengths")), page, s["selected"].shape[2], first, last)
    got = host(s["selected"])
    assert np.array_equal(host(s["selected_lengths"]), held)
    wrong = np.argwhere(got != want)
    assert not wrong.size, f"{len(wrong)} of {want.size}, the first at {wrong[0]}: {got[tuple(wrong[0])]} is not {want[tuple(wrong[0])]}"


PAGED = [0, 1, 15, 16, 17, 160, 161, 255, 256, 257, 1000, 1024, 1025, 3000]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("most,first,last", [(1, 0, 0), (1, 1, 0), (2, 1, 1), (5, 0, 2), (16, 1, 2), (17, 0, 0), (40, 20, 20), (64, 3, 0), (200, 1, 1)])
def test_selection_of_few_and_many_pages(dtype, most, first, last):
    check_select(select_case(PAGED, 4, 2, 64, 16, most, dtype, seed=most), 16, first, last)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [8, 16, 40, 72, 96, 128, 200, 256])
def test_selection_for_heads_of_any_size(dtype, dim):
    check_select(select_case([0, 90, 333, 700], 6, 3, dim, 8, 12, dtype, seed=dim), 8)


@pytest.mark.parametrize("hq,hk", [(1, 1), (5, 5), (7, 1), (16, 1), (17, 1), (32, 1), (66, 2)])
def test_selection_for_groups_of_any_size(hq, hk):
    check_select(select_case([40, 500, 123], hq, hk, 64, 8, 9, "bf16", seed=hq), 8)


@pytest.mark.parametrize("page", [1, 3, 24, 1000])
def test_selection_of_pages_of_any_size(page):
    check_select(select_case(np.array([0, 1, 9, 50, 77, 100, 333]) * page - np.array([0, 0, 1, 0, page - 1, 0, page // 2]), 4, 2, 16, page, 11, "f16", seed=page), page)


@pytest.mark.parametrize("pages", [2048, 2049, 5000, 8192, 8193, 20000])
def test_selection_among_many_pages(pages):
    # one request, whose scores several workgroups make, and more requests than workgroups are wanted for
    check_select(select_case([2 * pages - 1], 2, 1, 16, 2, 100, "bf16", seed=pages), 2)


@pytest.mark.parametrize("width", [100, 2100, 9000])
def test_selection_for_many_requests(width):
    rng = np.random.default_rng(width)
    lengths = rng.integers(0, 150, 600)
    lengths[17] = 4 * width
    check_select(select_case(lengths, 2, 2, 16, 4, 7, "f16", seed=width), 4)


@pytest.mark.parametrize("dtype,hq,hk,width", [("bf16", 2, 1, 100), ("f32", 1, 1, 700), ("f16", 5, 1, 2100), ("bf16", 3, 3, 65)])
def test_selection_of_rows_in_pieces_for_more_requests_than_a_workgroup_has_threads(dtype, hq, hk, width):
    rng = np.random.default_rng(width)
    lengths = rng.integers(0, 150, 300)
    lengths[::41] = 4 * rng.integers(1, width + 1, lengths[::41].shape)
    lengths[[0, 256, 299]] = 4 * width, 4 * width - 3, 4 * width
    s = select_case(lengths, hq, hk, 24, 4, 7, dtype, seed=width)
    check_select(s, 4)
    s["selected"].fill_(5), s["selected_lengths"].fill_(5)   # again in the same arrays
    check_select(s, 4)


def test_equal_scores_go_to_the_first_pages():
    for fill in (0.0, 1.5):
        s = select_case([700, 513, 16], 2, 2, 64, 8, 9, "bf16", seed=1)
        s["bounds"].fill_(fill)
        check_select(s, 8)
        check_select(s, 8, 0, 0)
    s = select_case([700, 513, 16], 2, 2, 64, 8, 9, "bf16", seed=1)
    s["bounds"].copy_(gpu(np.random.default_rng(2).integers(0, 2, tuple(s["bounds"].shape)).astype(np.float32)))
    s["q"].zero_()
    s["q"][:, :, 5] = 1.0                                    # two scores, 0 and 1, many pages each
    check_select(s, 8)
    s["q"][:, :, 5] = -1.0
    check_select(s, 8, 2, 3)
    s["bounds"].neg_()                                       # 0 and -0 among them
    check_select(s, 8, 0, 0)


def test_scores_that_are_not_finite_are_ordered_and_nan_comes_first():
    s = select_case([800, 800, 800, 800], 2, 2, 64, 8, 9, "bf16", seed=3)
    table = host(s["table"])
    for b in range(4):
        for at, x in ((3, math.nan), (40, math.inf), (41, -math.inf), (60, math.nan), (99, math.inf)):
            s["bounds"][int(table[b, at]), b % 2, 1, 7] = x
    s["bounds"][int(table[3, 50])] = -math.inf
    s["q"][1, :, 7] = 2.0
    s["q"][2, :, 9] = math.nan                               # every score is NaN
    check_select(s, 8)
    check_select(s, 8, 0, 0)


def test_scores_that_32_bits_cannot_tell_apart():
    # a large term that all pages share, and one that differs in the 30th bit
    s = select_case([900, 1600], 1, 1, 16, 8, 20, "f32", seed=4)
    s["q"].zero_()
    s["q"][:, :, 0], s["q"][:, :, 1] = 1.0, 1.0
    s["bounds"].zero_()
    s["bounds"][:, 0, 1, 0] = 4096.0
    s["bounds"][:, 0, 1, 1] = gpu(np.random.default_rng(4).permutation(s["bounds"].shape[0]).astype(np.float32)) * 2.0 ** -18
    check_select(s, 8)


def test_selection_leaves_out_pages_that_are_not_there():
    s = select_case([400, 400, 64, 400], 4, 2, 64, 8, 9, "bf16", seed=5)
    table = host(s["table"]).copy()
    table[0, ::3], table[1, :], table[2, 7], table[3, 49] = -1, 2 ** 31 - 1, s["bounds"].shape[0], -2 ** 31
    s["table"] = gpu(table)
    check_select(s, 8)
    check_select(s, 8, 4, 4)
    s["lengths"] = gpu(np.array([2 ** 31 - 1, -1, 10 ** 6, 399], np.int32))                # beyond the table
    check_select(s, 8)


def test_selection_of_nothing():
    import torch
    for lengths, most in (([], 4), ([0, 0], 4), ([100, 30], 0)):
        s = select_case(np.array(lengths, np.int32), 4, 2, 64, 8, most, "bf16", seed=6)
        check_select(s, 8, 0, 0)
    s = select_case([100, 30], 4, 2, 64, 8, 4, "bf16", seed=6)
    s["table"] = torch.zeros((2, 0), dtype=torch.int32, device="cuda")
    check_select(s, 8)


def test_selection_on_strided_tensors():
    import torch
    s = select_case([700, 100, 350], 4, 2, 64, 8, 9, "bf16", seed=7)
    q = torch.zeros((4, 3, 3, 64), dtype=torch.bfloat16, device="cuda")
    q[:, :, 1] = s["q"].transpose(0, 1)
    bounds = torch.full((2, s["bounds"].shape[0], 3, 72), math.nan, dtype=torch.bfloat16, device="cuda")
    bounds[:, :, 1:, :64] = s["bounds"].transpose(0, 1)
    table = torch.full((3, 200), -5, dtype=torch.int32, device="cuda")
    table[:, 1:1 + s["table"].shape[1]] = s["table"]
    selected, held = torch.full((2, 3, 20), 7, dtype=torch.int32, device="cuda"), torch.full((3, 5), 7, dtype=torch.int32, device="cuda")
    check_select({"q": q[:, :, 1].transpose(0, 1), "bounds": bounds[:, :, 1:, :64].transpose(0, 1), "table": table[:, 1:1 + s["table"].shape[1]],
                  "lengths": s["lengths"], "selected": selected[:, :, 4:13].transpose(0, 1), "selected_lengths": held[:, 1:3]}, 8)
    assert (selected[:, :, :4] == 7).all() and (selected[:, :, 13:] == 7).all() and (held[:, 0] == 7).all() and (held[:, 3:] == 7).all()


# --------------------------------------------------------------------------- attention over a table for each key head
def heads_case(lengths, hq, dim, page, dtype, seed, heads_first=False):
    """lengths [B, Hk]."""
    rng = np.random.default_rng(seed)
    lengths = np.asarray(lengths, np.int32)
    batch, hk = lengths.shape
    (table,), pages, used = pages_for(rng, page, lengths)
    caches = caches_of(rng, pages, page, hk, dim, dtype, used, heads_first)
    return {"q": gpu(rng.standard_normal((batch, hq, dim)).astype(np.float32), dtype), "k_cache": caches[0], "v_cache": caches[1], "table": gpu(table),
            "lengths": gpu(lengths)}


def attended(make, s, **kw):
    import torch
    out, lse = torch.full_like(s["q"], 7.0), torch.full(s["q"].shape[:2], 7.0, device="cuda")
    run([make(out=out, lse=lse, **s, **kw)])
    return host(out), host(lse)


def check_heads(s, dtype, window=0, scale=None):
    import paper_2407_13585_amd as fc
    dim = s["q"].shape[2]
    scale = dim ** -0.5 if scale is None else scale
    want = O.selected_attention(*(host(s[n]) for n in ("q", "k_cache", "v_cache", "table", "lengths")), scale, window)
    out, lse = attended(fc.PagedAttention, s, scale=scale, window=window)
    close(out, want, dtype, dim, lse=lse)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page", [1, 8, 16, 24, 64])
def test_attention_over_pages_of_each_key_head(dtype, page):
    rng = np.random.default_rng(page)
    lengths = rng.permutation([0, 0, 1, 15, 16, 17, 33, 64, 128, 129, 200, 700]).reshape(4, 3)
    check_heads(heads_case(lengths, 6, 64, page, dtype, seed=page, heads_first=page % 2 == 0), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hk,dim", [(1, 1, 40), (4, 4, 8), (34, 2, 64), (40, 2, 128), (6, 3, 256), (8, 2, 192)])
def test_attention_over_pages_of_each_key_head_for_heads_of_any_size_and_number(dtype, hq, hk, dim):
    lengths = np.random.default_rng(dim).integers(0, 300, (5, hk))
    check_heads(heads_case(lengths, hq, dim, 16, dtype, seed=dim), dtype)
    check_heads(heads_case(lengths, hq, dim, 16, dtype, seed=dim), dtype, window=50, scale=-0.3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_over_pages_of_each_key_head_of_long_and_of_many_short_rows(dtype):
    check_heads(heads_case([[5000, 0], [3, 2000]], 8, 128, 16, dtype, seed=1), dtype)
    check_heads(heads_case(np.random.default_rng(2).integers(0, 100, (400, 4)), 8, 64, 16, dtype, seed=2), dtype)


def test_attention_over_pages_of_each_key_head_of_no_requests_and_strided_tables():
    import torch
    check_heads(heads_case(np.zeros((0, 2), np.int32), 4, 64, 16, "bf16", seed=1), "bf16")
    s = heads_case([[100, 0, 40], [7, 300, 64]], 6, 64, 16, "bf16", seed=3)
    table, lengths = torch.full((3, 2, 40), -9, dtype=torch.int32, device="cuda"), torch.full((2, 5), 99, dtype=torch.int32, device="cuda")
    width = s["table"].shape[2]
    table[:, :, 2:2 + width] = s["table"].transpose(0, 1)
    lengths[:, 1:4] = s["lengths"]
    check_heads({**s, "table": table[:, :, 2:2 + width].transpose(0, 1), "lengths": lengths[:, 1:4]}, "bf16")


# --------------------------------------------------------------------------- prefixes
def prefix_case(groups, lengths, hq, hk, dim, page, dtype, seed, start=None, heads_first=False, sharp=1.0):
    """groups: (requests, keys of the prefix); requests behind the last one have none."""
    rng = np.random.default_rng(seed)
    lengths = np.asarray(lengths, np.int32)
    members, prefix = (np.array(x, np.int32) for x in zip(*groups)) if groups else (np.zeros(0, np.int32), np.zeros(0, np.int32))
    start = np.concatenate([[0], np.cumsum(members)]) if start is None else np.asarray(start)
    (prefix_table, table), pages, used = pages_for(rng, page, prefix, lengths)
    caches = caches_of(rng, pages, page, hk, dim, dtype, used, heads_first)
    return {"q": gpu(sharp * rng.standard_normal((len(lengths), hq, dim)).astype(np.float32), dtype), "k_cache": caches[0], "v_cache": caches[1],
            "prefix_table": gpu(prefix_table), "prefix_lengths": gpu(prefix), "group_start": gpu(start.astype(np.int32)), "table": gpu(table),
            "lengths": gpu(lengths)}


ORDER = ("q", "k_cache", "v_cache", "prefix_table", "prefix_lengths", "group_start", "table", "lengths")


def check_prefix(s, dtype, scale=None):
    import paper_2407_13585_amd as fc
    dim = s["q"].shape[2]
    scale = dim ** -0.5 if scale is None else scale
    want = O.prefix_attention(*(host(s[n]) for n in ORDER), scale)
    out, lse = attended(fc.PrefixAttention, s, scale=scale)
    close(out, want, dtype, dim, lse=lse)
    return out, lse


OWN = [0, 1, 5, 16, 17, 40, 100, 130, 33, 64]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page", [1, 8, 16, 24, 100])
def test_prefix_of_pages_of_any_size(dtype, page):
    check_prefix(prefix_case([(3, 100), (1, 64), (4, 257)], OWN, 4, 2, 64, page, dtype, seed=page, heads_first=page % 2 == 0), dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("prefix", [1, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 600])
def test_prefix_of_lengths_around_every_tile(dtype, prefix):
    for requests, hq in ((4, 4), (12, 8), (24, 16)):         # 8, 48 and 192 columns of two key heads: every number of columns a workgroup takes
        check_prefix(prefix_case([(requests, prefix)], np.arange(requests), hq, 2, 64, 16, dtype, seed=prefix), dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim", [8, 16, 40, 64, 72, 96, 128, 136, 192, 256])
def test_prefix_for_heads_of_any_size(dtype, dim):
    for requests in (3, 11, 40):
        check_prefix(prefix_case([(requests - 1, 150)], np.arange(requests) % 20, 8, 2, dim, 16, dtype, seed=dim), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hq,hk", [(1, 1), (5, 5), (7, 1), (33, 1), (66, 2), (130, 1)])
def test_prefix_for_groups_of_heads_of_any_size(dtype, hq, hk):
    check_prefix(prefix_case([(4, 90), (2, 200)], [3, 0, 50, 7, 1, 0, 20], hq, hk, 64, 16, dtype, seed=hq), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prefixes_that_are_long_or_many(dtype):
    check_prefix(prefix_case([(9, 6000)], [10, 0, 300] * 3, 8, 2, 128, 16, dtype, seed=1), dtype)
    check_prefix(prefix_case([(70, 900)], [3] * 70, 8, 2, 128, 16, dtype, seed=2), dtype)
    check_prefix(prefix_case([(2, n % 50) for n in range(150)], [n % 9 for n in range(310)], 4, 2, 64, 8, dtype, seed=3), dtype)
    check_prefix(prefix_case([(1, 5)] * 1024, [2] * 1030, 2, 1, 16, 8, dtype, seed=4), dtype)


@pytest.mark.parametrize("dtype,dim", [("f32", 40), ("f32", 128), ("f16", 64), ("bf16", 128), ("bf16", 96), ("f32", 256), ("f16", 256)])
def test_a_large_group_among_small_ones(dtype, dim):
    # as many columns as a small group has on average, and many times as many in one group
    groups = [(1, 70)] * 15 + [(40, 333)] + [(1, 129)] * 15
    check_prefix(prefix_case(groups, np.arange(75) % 23, 4, 1, dim, 8, dtype, seed=dim), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_groups_and_prefixes_that_are_empty(dtype):
    check_prefix(prefix_case([(3, 0), (0, 50), (2, 40), (0, 0)], OWN[:7], 4, 2, 64, 16, dtype, seed=1), dtype)
    check_prefix(prefix_case([(3, 0)], [0, 0, 0, 0], 4, 2, 64, 16, dtype, seed=2), dtype)
    check_prefix(prefix_case([(3, 70)], [0, 0, 0, 0], 4, 2, 64, 16, dtype, seed=3), dtype)
    check_prefix(prefix_case([(3, -70)], [5, -3, -2 ** 31], 4, 2, 64, 16, dtype, seed=3), dtype)
    check_prefix(prefix_case([], OWN, 4, 2, 64, 16, dtype, seed=4), dtype)
    check_prefix(prefix_case([(0, 30)], [], 4, 2, 64, 16, dtype, seed=5), dtype)


@pytest.mark.parametrize("start", [[2, 5, 9], [0, 0, 10], [-5, 4, 2 ** 31 - 1], [5, 3, 8], [9, 2, 1], [10, 10, 10], [-2 ** 31, -1, 0], [3, 20, 7]])
def test_starts_of_groups_of_any_kind(start):
    check_prefix(prefix_case([(5, 77), (5, 130)], OWN, 4, 2, 64, 16, "bf16", seed=6, start=start), "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prefix_skips_pages_that_are_not_there_and_lengths_beyond_the_table(dtype):
    s = prefix_case([(3, 200), (3, 100), (3, 64)], OWN, 4, 2, 64, 16, dtype, seed=7)
    table, own = host(s["prefix_table"]).copy(), host(s["table"]).copy()
    table[0, 2], table[1, :], table[2, 3], own[5, 1], own[4, :] = -1, 2 ** 31 - 1, s["k_cache"].shape[0], -2 ** 31, -3
    s["prefix_table"], s["table"] = gpu(table), gpu(own)
    check_prefix(s, dtype)
    s["k_cache"], s["v_cache"] = (c.nan_to_num(0.5, 0.25, -0.25) for c in (s["k_cache"], s["v_cache"]))
    s["prefix_lengths"] = gpu(np.array([10 ** 9, 2 ** 31 - 1, 64], np.int32))
    check_prefix(s, dtype)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_prefix_with_large_scores(dtype):
    s = prefix_case([(5, 300), (4, 70)], OWN, 4, 2, 64, 16, dtype, seed=8, sharp=40.0)
    check_prefix(s, dtype)
    check_prefix(s, dtype, scale=-3.0)
    check_prefix(s, dtype, scale=0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prefix_of_keys_and_values_that_are_not_finite(dtype):
    s = prefix_case([(4, 90), (4, 90)], [40] * 10, 2, 2, 64, 16, dtype, seed=9)
    clean = check_prefix(s, dtype)
    table, own = host(s["prefix_table"]), host(s["table"])
    s["k_cache"][int(table[0, 1]), 3, 0, 5] = math.nan
    s["v_cache"][int(table[1, 2]), 7, 1, 9] = math.inf
    s["v_cache"][int(own[8, 0]), 0, 0, 2] = -math.inf
    import paper_2407_13585_amd as fc
    out, lse = attended(fc.PrefixAttention, s)
    changed = np.zeros(out.shape, bool)
    changed[:4, 0] = changed[4:8, 1, 9] = changed[8, 0, 2] = True
    assert np.isnan(out[:4, 0]).all() and np.isnan(lse[:4, 0]).all() and (out[4:8, 1, 9] == math.inf).all() and out[8, 0, 2] == -math.inf
    assert np.array_equal(out[~changed], clean[0][~changed])


@pytest.mark.parametrize("dtype,page", [("f32", 16), ("f16", 5), ("bf16", 16)])
def test_prefix_whose_scores_are_all_minus_infinity_is_as_none(dtype, page):
    s = prefix_case([(4, 90)], [0, 40, 3, 17, 5], 2, 1, 64, page, dtype, seed=10)
    s["q"].abs_()
    for p in host(s["prefix_table"])[0][:-(-90 // page)]:
        s["k_cache"][int(p)] = -math.inf
    check_prefix(s, dtype)


def test_prefix_is_as_exact_as_attention_over_the_whole_of_each_request():
    # one table a request, the prefix' pages first: the same keys, so the same result but for the order of sums
    import torch
    import paper_2407_13585_amd as fc
    s = prefix_case([(6, 320)], [0, 1, 5, 16, 40, 100], 8, 2, 128, 16, "f32", seed=11)
    n = 20
    whole = {**{k: s[k] for k in ("q", "k_cache", "v_cache")}, "table": torch.cat([s["prefix_table"][:, :n].expand(6, n), s["table"]], 1).contiguous(),
             "lengths": s["lengths"] + 320}
    (out, lse), (ref, ref_lse) = attended(fc.PrefixAttention, s), attended(fc.PagedAttention, whole)
    near(out, ref, 2.0 ** -17)
    near(lse, ref_lse, 2.0 ** -18)


def test_prefix_on_strided_tensors_and_without_lse():
    import torch
    import paper_2407_13585_amd as fc
    s = prefix_case([(2, 100), (3, 70)], [5, 70, 129, 0, 3, 9], 6, 2, 64, 16, "bf16", seed=12)
    want = O.prefix_attention(*(host(s[n]) for n in ORDER), 0.125)
    wide = torch.zeros((6, 6, 3, 64), dtype=torch.bfloat16, device="cuda")
    wide[:, :, 1] = s["q"]
    tables = torch.full((2, 40), -5, dtype=torch.int32, device="cuda")
    tables[:, 1:1 + s["prefix_table"].shape[1]] = s["prefix_table"]
    out = torch.full((6, 6, 65), 9.0, dtype=torch.bfloat16, device="cuda")
    run([fc.PrefixAttention(out=out[:, :, 1:], **{**s, "q": wide[:, :, 1], "prefix_table": tables[:, 1:1 + s["prefix_table"].shape[1]]})])
    close(host(out[:, :, 1:]), want, "bf16", 64)
    assert (out[:, :, 0] == 9).all()
    check_prefix({**s, "q": s["q"][:1].expand(6, 6, 64)}, "bf16")


def test_results_have_the_same_bits_every_time():
    import paper_2407_13585_amd as fc
    s = prefix_case([(9, 3000), (3, 500)], [10, 0, 300] * 5, 8, 2, 128, 16, "bf16", seed=13)
    first = attended(fc.PrefixAttention, s)
    for _ in range(3):
        assert all(np.array_equal(a, b) for a, b in zip(first, attended(fc.PrefixAttention, s)))


@pytest.mark.parametrize("heads_first", [False, True])
def test_everything_beyond_32_bit_offsets(heads_first):
    # caches and bounds of more than 2^32 elements together with their strides: the pages in use lie at the far end
    import torch
    import paper_2407_13585_amd as fc
    pages, page, hk, dim = (1 << 32) // (16 * 2 * 64) + 9, 16, 2, 64
    shape = (pages, hk, page, dim) if heads_first else (pages, page, hk, dim)
    gen = torch.Generator("cuda").manual_seed(2)
    caches = []
    for _ in range(2):
        c = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        c[-9:] = torch.randn(c[-9:].shape, device="cuda", generator=gen).to(torch.bfloat16)
        caches.append(c.transpose(1, 2) if heads_first else c)
    store = torch.empty((pages, 16 * hk * dim), dtype=torch.bfloat16, device="cuda")       # rows as far apart as the cache's pages
    bounds = store[:, :hk * 2 * dim].view(pages, hk, 2, dim)
    far = np.array([[pages - 1, pages - 5, pages - 3, pages - 7]], np.int32)
    table, lengths = gpu(far), gpu(np.array([60], np.int32))
    q = torch.randn((1, 4, dim), device="cuda", generator=gen).to(torch.bfloat16)
    selected, held = torch.zeros((1, hk, 3), dtype=torch.int32, device="cuda"), torch.zeros((1, hk), dtype=torch.int32, device="cuda")
    outs, lses = [torch.empty_like(q) for _ in range(2)], [torch.empty((1, 4), device="cuda") for _ in range(2)]
    run([fc.PageBounds(k_cache=caches[0], table=table, lengths_before=torch.zeros_like(lengths), lengths=lengths, bounds=bounds),
         fc.PageSelect(q=q, bounds=bounds, table=table, lengths=lengths, page_size=page, selected=selected, selected_lengths=held),
         fc.PagedAttention(q=q, k_cache=caches[0], v_cache=caches[1], table=selected, lengths=held, out=outs[0], lse=lses[0]),
         fc.PrefixAttention(q=q, k_cache=caches[0], v_cache=caches[1], prefix_table=table[:, 1:], prefix_lengths=gpu(np.array([40], np.int32)),
                            group_start=gpu(np.array([0, 1], np.int32)), table=table[:, :1], lengths=gpu(np.array([9], np.int32)), out=outs[1], lse=lses[1])])
    base = pages - 9
    small = [host(c[-9:]) for c in caches]
    near_bounds = O.page_bounds(small[0], far - base, [0], [60], np.zeros((9, hk, 2, dim)))
    assert np.array_equal(host(bounds[-9:])[far[0] - base], near_bounds[far[0] - base])
    want, want_held = O.page_select(host(q), near_bounds, far - base, [60], page, 3, 1, 1)
    assert np.array_equal(host(selected) - base, want) and np.array_equal(host(held), want_held)
    close(host(outs[0]), O.selected_attention(host(q), *small, want, want_held, dim ** -0.5), "bf16", dim, lse=host(lses[0]))
    close(host(outs[1]), O.prefix_attention(host(q), *small, far[:, 1:] - base, [40], [0, 1], far[:, :1] - base, [9], dim ** -0.5), "bf16", dim, lse=host(lses[1]))
    del caches, bounds, store
    torch.cuda.empty_cache()


# --------------------------------------------------------------------------- together
def test_a_step_over_selected_pages_and_one_over_a_prefix_replay_from_a_graph():
    """Pages given out, a new key appended, its page's bounds, a selection and attention over it; beside it all requests as readers of one prefix.
    Several replays, lengths that grow, each against the eager step and the oracle; attention over all pages where they are few."""
    import torch
    import paper_2407_13585_amd as fc
    batch, hq, hk, dim, page, width, pages, most = 5, 8, 2, 64, 8, 16, 96, 5
    rng = np.random.default_rng(4)
    lengths = np.array([0, 7, 30, 60, 100], np.int32)
    have = -(-lengths // page)
    order = rng.permutation(pages).astype(np.int32)
    prefix_pages, order = order[:6], order[6:]
    table = np.full((batch, width), -1, np.int32)
    table[np.arange(width)[None, :] < have[:, None]] = order[:have.sum()]
    free = order[have.sum():]
    pool = np.concatenate([free, np.zeros(pages - free.size, np.int32)]).astype(np.int32)
    angle = rng.uniform(-3, 3, (200, dim // 2))
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    t = {"lengths": gpu(lengths), "new": gpu(np.ones(batch, np.int32)), "pool": gpu(pool), "cursor": gpu(np.array([0, free.size], np.int64)), "table": gpu(table),
         "after": i32(batch), "row": i32(batch + 1), "slots": gpu(np.zeros(batch, np.int64)), "positions": i32(batch), "request": i32(batch),
         "cursor_after": gpu(np.zeros(2, np.int64)), "unplaced": gpu(np.zeros(1, np.int64)), "selected": i32(batch, hk, most), "held": i32(batch, hk),
         "cos_sin": gpu(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)), "w": gpu(np.ones(dim, np.float32), "bf16")}
    for n, heads in (("q", hq), ("k", hk), ("v", hk)):
        t[n] = torch.zeros((batch, heads, dim), dtype=torch.bfloat16, device="cuda")
    for n in ("q_out", "out", "shared"):
        t[n] = torch.empty_like(t["q"])
    caches = [gpu(rng.standard_normal((pages, page, hk, dim)).astype(np.float32), "bf16") for _ in range(2)]
    t["bounds"] = torch.empty((pages, hk, 2, dim), dtype=torch.bfloat16, device="cuda")
    # bounds of what is there before the first step
    run([fc.PageBounds(k_cache=caches[0], table=t["table"], lengths_before=torch.zeros_like(t["lengths"]), lengths=t["lengths"], bounds=t["bounds"])])
    ops = [fc.PageMap(page_size=page, lengths=t["lengths"], new_tokens=t["new"], pool=t["pool"], cursor=t["cursor"], table=t["table"],
                      lengths_after=t["after"], row_start=t["row"], slots=t["slots"], positions=t["positions"], request=t["request"],
                      cursor_after=t["cursor_after"], unplaced=t["unplaced"]),
           fc.HeadNormRope(q=t["q"], k=t["k"], v=t["v"], q_out=t["q_out"], k_cache=caches[0], v_cache=caches[1], slots=t["slots"], q_weight=t["w"],
                           k_weight=t["w"], cos_sin=t["cos_sin"], positions=t["positions"].view(1, -1)),
           fc.PageBounds(k_cache=caches[0], table=t["table"], lengths_before=t["lengths"], lengths=t["after"], bounds=t["bounds"]),
           fc.PageSelect(q=t["q_out"], bounds=t["bounds"], table=t["table"], lengths=t["after"], page_size=page, selected=t["selected"], selected_lengths=t["held"]),
           fc.PagedAttention(q=t["q_out"], k_cache=caches[0], v_cache=caches[1], table=t["selected"], lengths=t["held"], out=t["out"]),
           fc.PrefixAttention(q=t["q_out"], k_cache=caches[0], v_cache=caches[1], prefix_table=gpu(prefix_pages[None]), prefix_lengths=gpu(np.array([45], np.int32)),
                              group_start=gpu(np.array([0, batch - 1], np.int32)), table=t["table"], lengths=t["after"], out=t["shared"])]
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
    for step in range(4):
        for n in "qkv":
            t[n].copy_(gpu(rng.standard_normal(tuple(t[n].shape)).astype(np.float32), "bf16"))
        torch.cuda.synchronize()
        bounds_before = host(t["bounds"])
        graph.replay()
        torch.cuda.synchronize()
        names = ("after", "slots", "q_out", "out", "shared", "table", "pool", "selected", "held", "bounds")
        got = {n: host(t[n]) for n in names}
        for n in ("q_out", "out", "shared", "slots", "selected", "held"):
            t[n].fill_(3)
        fc.fc_run_operators(ops, scratch, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert all(np.array_equal(got[n], host(t[n]), equal_nan=n == "bounds") for n in names), step      # bounds of unused pages are anything
        k, v = (host(c) for c in caches)
        in_use = np.concatenate([got["table"][b, :-(-n // page)] for b, n in enumerate(got["after"])])
        want = O.page_bounds(k, got["table"], host(t["lengths"]), got["after"], bounds_before)
        assert np.array_equal(got["bounds"][in_use], want[in_use])
        selected, held = O.page_select(got["q_out"], want, got["table"], got["after"], page, most, 1, 1)
        assert np.array_equal(got["selected"], selected) and np.array_equal(got["held"], held)
        close(got["out"], O.selected_attention(got["q_out"], k, v, selected, held, dim ** -0.5), "bf16", dim)
        few = got["after"] <= most * page
        close(got["out"][few], [x[few] for x in O.paged_attention(got["q_out"], k, v, got["table"], got["after"], dim ** -0.5)], "bf16", dim)
        close(got["shared"], O.prefix_attention(got["q_out"], k, v, prefix_pages[None], [45], [0, batch - 1], got["table"], got["after"], dim ** -0.5), "bf16", dim)
        t["lengths"].copy_(t["after"])
        t["cursor"].copy_(t["cursor_after"])
        fc.fc_check(scratch)


def test_the_operators_run_on_the_stream_they_are_given_two_at_a_time():
    # two streams, each with a scratch buffer of its own
    import torch
    import paper_2407_13585_amd as fc
    cases = [prefix_case([(9, 2000), (3, 500)], [10, 0, 300] * 5, 8, 2, 128, 16, "bf16", seed=k) for k in (14, 15)]
    want = [attended(fc.PrefixAttention, s) for s in cases]
    streams, kept = [torch.cuda.Stream() for _ in cases], []
    for s in cases:
        out, lse = torch.full_like(s["q"], 7.0), torch.full(s["q"].shape[:2], 7.0, device="cuda")
        ops = [fc.PrefixAttention(out=out, lse=lse, **s)]
        kept.append((out, lse, fc.BoundOperators(ops, torch.zeros(fc.fc_operators_scratch_bytes(ops), dtype=torch.uint8, device="cuda"))))
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, (_, _, bound) in zip(streams, kept):
            bound(stream.cuda_stream)
    torch.cuda.synchronize()
    for (out, lse, _), (ref, ref_lse) in zip(kept, want):
        assert np.array_equal(host(out), ref) and np.array_equal(host(lse), ref_lse)
