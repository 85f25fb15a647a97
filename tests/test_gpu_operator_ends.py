"""The operators of a serving cache at the ends of their ranges, against the definitions in 64 bits (oracle/cache.py).
Tolerances are those of test_gpu_operators.py unless a test says otherwise."""
import numpy as np
import pytest

from test_gpu_operators import LENGTHS, TINY, U, attention_case, attention_raw, attention_want, check_attention, check_grad, check_heads, gpu, heads_case, host, near, run, types

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("axes", [1, 3])
@pytest.mark.parametrize("dim,rotary", [(64, 64), (64, 32), (72, 18), (30, 30)])
def test_every_position_is_outside_a_table_of_angles_without_rows(dtype, axes, dim, rotary):
    # whatever the way to the angles: the rotated elements are NaN, the others as without a rotation, and so are gradients
    import torch
    s = heads_case(37, 5, 2, dim, rotary, dtype, seed=dim, axes=axes)
    s["cos_sin"] = torch.empty((0, rotary), device="cuda")
    for interleaved in (False, True):
        check_heads(s, dtype, interleaved=interleaved)
        check_grad(s, dtype, interleaved=interleaved)
        check_grad(s, dtype, interleaved=interleaved, weight=False)


def test_pages_are_entered_for_more_tokens_than_can_be_counted_where_every_counted_one_has_a_place():
    # two requests ask for 2^31-1 tokens each, and there are places for 2^31-1: those of the first
    import torch
    import paper_2407_13585_amd as fc
    page, most = 1 << 22, 2 ** 31 - 1
    pages = 2 * 512
    order = np.random.default_rng(5).permutation(pages).astype(np.int32)
    i32 = dict(dtype=torch.int32, device="cuda")
    table, after, row = torch.full((2, 600), -1, **i32), torch.zeros(2, **i32), torch.zeros(3, **i32)
    slots, positions, request = torch.empty(most, dtype=torch.int64, device="cuda"), torch.empty(most, **i32), torch.empty(most, **i32)
    cursor_after, unplaced = (torch.zeros(n, dtype=torch.int64, device="cuda") for n in (2, 1))
    run([fc.PageMap(page_size=page, lengths=torch.zeros(2, **i32), new_tokens=torch.full((2,), most, **i32), pool=gpu(order),
                    cursor=gpu(np.array([0, pages], np.int64)), table=table, lengths_after=after, row_start=row, slots=slots, positions=positions,
                    request=request, cursor_after=cursor_after, unplaced=unplaced)])
    want = np.full((2, 600), -1, np.int32)
    want[:, :512] = order.reshape(2, 512)
    assert np.array_equal(host(table), want)
    assert host(after).tolist() == [most, most] and host(row).tolist() == [0, most, most]
    assert host(cursor_after).tolist() == [pages, pages] and host(unplaced)[0] == 0
    for at in (torch.arange(0, most, 9973, device="cuda"), torch.arange(most - 5000, most, device="cuda")):
        assert torch.equal(positions[at].long(), at) and bool((request[at] == 0).all())
        assert torch.equal(slots[at], gpu(order)[at // page].long() * page + at % page)
    del slots, positions, request
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,large", [("f32", 1e30), ("f16", 60000.0), ("bf16", 1e35)])
@pytest.mark.parametrize("page", [16, 5])
@pytest.mark.parametrize("below", [40.0, 100.0])
def test_keys_of_no_weight_to_speak_of_add_nothing_however_many_they_are(dtype, large, page, below):
    # One key has all the weight, each of the others e^-below of it.  Where that is too little for the type's numbers they must add nothing: together they
    # come to 20000 * e^-40 * 6e4 = 5e-9 for f16, 20000 * e^-100 * 1e35 = 7e-5 for bf16, and to less for f32.
    import torch
    keys, dim = 20000, 64
    if below == 40.0 and dtype != "f16":
        large = 1e6                                              # 20000 * e^-40 * 1e6 = 8e-8
    pages = -(-keys // page)
    k = torch.zeros((pages * page, 1, dim), device="cuda")
    v = torch.full((pages * page, 1, dim), large, device="cuda")
    k[:, 0, 0] = -below
    at = 12345
    k[at, 0, 0], v[at] = 0.0, 1.0
    q = torch.zeros((1, 2, dim), device="cuda")
    q[:, :, 0] = 8.0                                             # times the scale of 1/8: scores of 0 and -below
    s = {"q": q.to(types()[dtype]), "k_cache": k.view(pages, page, 1, dim).to(types()[dtype]), "v_cache": v.view(pages, page, 1, dim).to(types()[dtype]),
         "table": torch.arange(pages, dtype=torch.int32, device="cuda")[None], "lengths": gpu(np.array([keys], np.int32))}
    check_attention(s, dtype)


def test_keys_of_no_weight_in_one_wave_s_row_add_nothing_in_16_bits():
    # 1024 requests of 65536 keys over the same two pages, so that a wave walks 16384 keys after the one that has all the weight.  2^-38 of it for each
    # of them, the smallest weight that 16 bits hold here, would make 1 + 16384 * 2^-38 * 6e4 = 1.0036 of a result that is 1.
    import torch
    import paper_2407_13585_amd as fc
    requests, keys, page, dim = 1024, 65536, 16, 64
    half = dict(dtype=torch.float16, device="cuda")
    k, v = torch.zeros((2, page, 1, dim), **half), torch.full((2, page, 1, dim), 6e4, **half)
    k[..., 0] = -100.0
    k[1, 0], v[1, 0] = 0.0, 1.0
    table = torch.zeros((requests, keys // page), dtype=torch.int32, device="cuda")
    table[:, 0] = 1
    q, out, lse = torch.zeros((requests, 1, dim), **half), torch.empty((requests, 1, dim), **half), torch.empty((requests, 1), device="cuda")
    q[..., 0] = 8.0
    run([fc.PagedAttention(q=q, k_cache=k, v_cache=v, table=table, lengths=torch.full((requests,), keys, dtype=torch.int32, device="cuda"), out=out, lse=lse)])
    assert bool((out == 1).all()) and bool((lse == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("dim,page,window", [(8, 16, 0), (64, 16, 0), (64, 7, 90), (80, 24, 0), (96, 24, 200), (128, 32, 0), (128, 3, 0), (192, 16, 0), (256, 5, 0)])
def test_attention_holds_weights_in_more_than_16_bits(dtype, dim, page, window):
    # check_attention allows every type what bf16 needs, 2^-16 of a weight.  f32 has its weights in full and f16 in 22 bits: what is left is the error of
    # the scores and 2^-20 for powers and sums, twice, and the result's own rounding.
    s = attention_case(LENGTHS + [3000], 6, 3, dim, page, dtype, seed=dim + page)
    out, _ = check_attention(s, dtype, window=window)
    ref, _, reach, spread = attention_want(s, dim ** -0.5, window)
    weight = (dim + 8) * 2.0 ** -24 * reach[..., None] + 2.0 ** -20 + (2.0 ** -22 if dtype == "f16" else 0.0)
    near(out, ref, 2 * weight * spread + U[dtype] * np.abs(ref) + TINY[dtype], "out")


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("page", [16, 5])
def test_scores_that_are_all_minus_infinity_leave_what_no_keys_leave(dtype, page):
    # one element of every key of requests 0 and 1, whose key head is 0, is infinite and that of its queries negative; the other heads keep their keys
    s = attention_case([1, 700, 700], 4, 2, 64, page, dtype, seed=page)
    q = s["q"]
    q[:2, :2, 3] = -abs(q[:2, :2, 3]) - 1
    table = host(s["table"])
    for b, n in ((0, 1), (1, 700)):
        for j in range(n):
            s["k_cache"][int(table[b, j // page]), j % page, 0, 3] = float("inf")
    before = attention_want({**s, "k_cache": s["k_cache"].nan_to_num(posinf=0.0), "v_cache": s["v_cache"].nan_to_num()}, 0.125, 0)
    out, lse = (host(t) for t in attention_raw(s))
    assert (out[:2, :2] == 0).all() and (lse[:2, :2] == -np.inf).all()
    for b, h in ((0, 2), (0, 3), (1, 2), (1, 3), (2, 0), (2, 1), (2, 2), (2, 3)):
        near(out[b, h], before[0][b, h], 2.0 ** -7 if dtype != "f32" else 1e-4)
        near(lse[b, h:h + 1], before[1][b, h:h + 1], 1e-4)


def test_operators_share_the_scratch_of_a_segmented_fold_of_as_many_rows_as_its_flags_allow():
    # 66.5 million rows, an element in every sixteenth: the column-blocked fold's flags reach into the operators' counters, which are left cleared
    import torch
    import paper_2407_13585_amd as fc
    from paper_2407_13585_amd import binding as B
    from test_operator_limits import spmv_of_many_rows
    rows, cols = 66500000, 1500000
    elements = -(-rows // 16)
    g, part = spmv_of_many_rows(rows, elements, cols)
    assert "column-blocked" in fc.fc_cluster_kernel(g, part, 0)
    gen = torch.Generator("cuda").manual_seed(1)
    x, vals = (torch.rand(n, generator=gen, device="cuda") + 0.5 for n in (cols, elements))
    col = torch.randint(0, cols, (elements,), generator=gen, device="cuda", dtype=torch.int32)
    off = ((torch.arange(rows + 1, device="cuda") + 15) // 16).int()
    y, want = torch.empty(rows, device="cuda"), torch.zeros(rows, device="cuda")
    want[::16] = vals * x[col.long()]
    scratch = torch.zeros(fc.fc_scratch_bytes(g, part), dtype=torch.uint8, device="cuda")
    fold = B.BoundRun(g, part, {"x": x, "col": col, "vals": vals, "off": off, "y": y}, scratch)
    s = attention_case([5000, 900], 4, 2, 64, 16, "f32", seed=1)
    out, lse = torch.empty((2, 4, 64), device="cuda"), torch.empty((2, 4), device="cuda")
    attend = fc.BoundOperators([fc.PagedAttention(out=out, lse=lse, **s)], scratch)
    ref, ref_lse, _, _ = attention_want(s, 0.125, 0)
    for _ in range(3):
        for t in (y, out, lse):
            t.fill_(7.0)
        fold(torch.cuda.current_stream().cuda_stream)
        attend(torch.cuda.current_stream().cuda_stream)
        fc.fc_check(scratch, torch.cuda.current_stream().cuda_stream)
        assert torch.equal(y, want)
        near(host(out), ref, 1e-5)
        near(host(lse), ref_lse, 1e-5)
