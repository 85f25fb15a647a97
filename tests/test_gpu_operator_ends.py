"""The operators of a serving cache at the ends of their ranges, against the definitions in 64 bits (oracle/cache.py).
Tolerances are those of test_gpu_operators.py unless a test says otherwise."""
import pytest

from test_gpu_operators import check_grad, check_heads, heads_case

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
