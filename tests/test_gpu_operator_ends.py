"""The operators of a serving cache at the ends of their ranges, against the definitions in 64 bits (oracle/cache.py).
Tolerances are those of test_gpu_operators.py unless a test says otherwise."""
import numpy as np
import pytest

from test_gpu_operators import check_grad, check_heads, gpu, heads_case, host, run

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
