"""Attention over shared prefixes (fc_prefix_attention) where scores are so large that 32 bits hold them to no more than whole steps, on the GPU against the
definition in 64 bits (oracle/cache.py).

A few keys lead, and every request sees one at least: they are equal, and their products with every query are sums of equal powers of 2, so that nothing of
a product is rounded, whatever its size.  All other keys lie behind them by far more than any weight reaches.  So the result is the mean of the leaders' values, and the rounding of a large
score, which is the same for all of them, must not show in it: what is left are the weights, 2^-20 for the power of 2 and 2^-16 for the bits that a weight is
held in, once in the sum above and once in the one below, and half a step of the result.  lse is a score: its product with the scale and the scale itself are rounded
(2 * 2^-24), and so is the sum with the logarithm (2^-24); 2^-22 of it, and 2^-20 for the logarithm."""
import math

import numpy as np
import pytest

from oracle import cache as O
from test_gpu_operators import TINY, U, gpu, host, near
from test_gpu_selection_and_prefix import ORDER, attended, check_prefix, prefix_case

pytestmark = pytest.mark.gpu

PAGE = 16


def leaders_case(dtype, size, members, prefix, own, places, hq, hk, dim, seed, opposed=False):
    """Keys and queries whose products are dim * size at most, size a power of 2; places: (pages of a group's prefix or of a request, key), of each leader.
    opposed: the other keys are the leaders' negatives, not random ones."""
    s = prefix_case([(members, prefix)], own, hq, hk, dim, PAGE, dtype, seed)
    rng = np.random.default_rng(seed)
    sign = rng.choice([-1.0, 1.0], (hk, dim)).astype(np.float32)
    a, b = 2.0 ** (math.log2(size) // 2), size / 2.0 ** (math.log2(size) // 2)
    times = rng.choice([0.5, 1.0], (len(own), hq, 1)).astype(np.float32)
    s["q"] = gpu(np.float32(a) * np.repeat(sign, hq // hk, 0)[None] * times, dtype)
    s["k_cache"] = s["k_cache"] * 2.0 ** -6 * b              # behind by most of the score
    if opposed:
        s["k_cache"].copy_(gpu(np.float32(-b) * sign, dtype))
    for table, row, j in places:
        s["k_cache"][int(s[table][row, j // PAGE]), j % PAGE] = gpu(np.float32(b) * sign, dtype)
    return s


def check_leaders(s, dtype, scale):
    import torch
    import paper_2407_13585_amd as fc
    ref, logs, _, spread = O.prefix_attention(*(host(s[n]) for n in ORDER), scale)
    tol = 2 * (2.0 ** -20 + 2.0 ** -16) * spread + U[dtype] * np.abs(ref) + TINY[dtype]
    log_tol = 2.0 ** -22 * np.abs(np.where(np.isfinite(logs), logs, 0.0)) + 2.0 ** -20
    out, lse = attended(fc.PrefixAttention, s, scale=scale)
    near(out, ref, tol, "out")
    near(lse, logs, log_tol, "lse")
    # one table a request, the prefix' pages first
    n = int(s["prefix_lengths"][0])
    if n % PAGE == 0:
        batch, pages = s["q"].shape[0], n // PAGE
        members = int(s["group_start"][1])
        whole = torch.cat([s["prefix_table"][:1, :pages].expand(batch, pages), s["table"]], 1)
        whole[members:, :s["table"].shape[1]] = s["table"][members:]
        lengths = s["lengths"].clone()
        lengths[:members] += n
        out, lse = attended(fc.PagedAttention, {**{k: s[k] for k in ("q", "k_cache", "v_cache")}, "table": whole.contiguous(), "lengths": lengths}, scale=scale)
        near(out, ref, tol, "out of one table a request")
        near(lse, logs, log_tol, "lse of one table a request")


SIZES = [("f16", 2.0 ** n) for n in (18, 21, 23, 25, 27, 28)] + [("bf16", 2.0 ** n) for n in (18, 25, 27, 31, 57, 90, 110)] + [("f32", 2.0 ** n) for n in (18, 27, 57, 110)]


@pytest.mark.parametrize("dtype,size", SIZES)
@pytest.mark.parametrize("scale", [0.125, 64 ** -0.5 * 1.1, -0.3])
def test_one_key_leads_by_scores_of_any_size(dtype, size, scale):
    outside = [("table", 8, 25)]                             # of the request that has no prefix
    for own, places in (([0, 1, 40, 0, 17, 64, 3, 100, 50], [("prefix_table", 0, 7)] + outside),
                        ([0, 1, 40, 0, 17, 64, 3, 100, 50], [("prefix_table", 0, 319)] + outside),
                        ([5, 1, 40, 9, 17, 64, 3, 100, 50], [("table", b, b // 2) for b in (0, 2, 3, 4, 5, 6, 7)] + [("table", 1, 0)] + outside)):
        s = leaders_case(dtype, size, 8, 320, own, places, 4, 2, 64, seed=3)
        if scale < 0:
            s["q"].neg_()
        check_leaders(s, dtype, scale)


@pytest.mark.parametrize("dtype,size", SIZES)
@pytest.mark.parametrize("dim,hq,hk", [(64, 8, 2), (96, 4, 2), (128, 8, 4), (192, 6, 2), (256, 4, 4)])
def test_equal_keys_of_a_prefix_and_behind_it_weigh_the_same_whatever_their_score(dtype, size, dim, hq, hk):
    # in one unit, in those of other waves and workgroups, and among the requests' own keys; few and many columns
    size /= 2 ** math.ceil(math.log2(dim / 64))
    for members in (3, 8, 24, 50):
        own = [n % 90 for n in range(7, 7 + 11 * members, 11)] + [45]                      # the last one has no prefix
        places = [("prefix_table", 0, j) for j in (0, 1, 40, 77, 500, 1111, 1999)]
        places += [("table", b, n // 2) for b, n in enumerate(own) if b == members or (n > 20 and b % 3)]
        check_leaders(leaders_case(dtype, size, members, 2000, own, places, hq, hk, dim, seed=members), dtype, dim ** -0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1.9, -1.9, 1.0, 2.0 ** -20, 2.0 ** -120, 2.0 ** -125, 2.0 ** -126, 2.0 ** -127])
def test_products_at_both_ends_of_32_bits(dtype, scale):
    # products of 2^127 and of -2^127, whose difference is infinite: scores of 1.9 * 2^127 at most, and of 1 and less, where all keys weigh something (a scale of
    # 2^-127 times the logarithm's base is off by 2^-23, and an exponent of 2.9 so by less than 2^-21)
    own = [0, 1, 40, 9, 17, 64, 3, 100, 45]
    places = [("prefix_table", 0, j) for j in (3, 150, 319)] + [("table", 2, 30), ("table", 7, 99), ("table", 8, 25)]
    s = leaders_case(dtype, 2.0 ** 121, 8, 320, own, places, 4, 2, 64, seed=5, opposed=True)
    if scale < 0:
        s["q"].neg_()
    check_leaders(s, dtype, scale)


@pytest.mark.parametrize("scale", [2.0 ** 3, -(2.0 ** 40)])
def test_scores_beyond_32_bits_are_infinite_as_without_a_prefix(scale):
    import paper_2407_13585_amd as fc
    own = [0, 1, 40, 9, 17, 64, 3, 100, 45]
    places = [("prefix_table", 0, j) for j in (3, 150, 319)] + [("table", 2, 30), ("table", 7, 99), ("table", 8, 25)]
    for leaders in (places, []):
        s = leaders_case("bf16", 2.0 ** 121, 8, 320, own, leaders, 4, 2, 64, seed=5, opposed=True)
        if scale < 0:
            s["q"].neg_()
        out, lse = attended(fc.PrefixAttention, s, scale=scale)
        if leaders:                                          # the largest is infinite
            assert np.isnan(out).all() and np.isnan(lse).all()
        else:                                                # all are -inf: as no keys
            assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_a_scale_of_zero_over_prefixes_of_which_nothing_is_there(dtype):
    # every score is 0, so out is the mean of the values that are there, and lse the logarithm of their number
    s = prefix_case([(3, 100), (3, 64), (2, 40)], [0, 5, 40, 0, 7, 64, 0, 3, 9], 8, 2, 64, PAGE, dtype, seed=6)
    table = host(s["prefix_table"]).copy()
    table[0, :], table[2, 1] = -1, 2 ** 31 - 1
    s["prefix_table"] = gpu(table)
    check_prefix(s, dtype, scale=0.0)
    check_prefix(s, dtype, scale=-0.0)
