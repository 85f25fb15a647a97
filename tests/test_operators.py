"""The operators of a serving cache without a GPU: what they refuse before anything is enqueued, the layout of their structs, and the
oracle they are compared with on the GPU."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest

import paper_2407_13585_amd as fc
from oracle import cache as O
from paper_2407_13585_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SCRATCH = (0x10000000, 1 << 30)               # like every address here: nothing is enqueued, so it is never used


class Device:
    type = "cuda"


class T:
    """What the binding asks of a torch tensor."""

    device = Device()

    def __init__(self, dtype, *shape, stride=None, ptr=0x20000000):
        self.dtype, self.shape, self.ptr = "torch." + dtype, shape, ptr
        self.strides = stride or tuple(int(np.prod(shape[k + 1:], dtype=np.int64)) for k in range(len(shape)))

    def data_ptr(self):
        return self.ptr

    def dim(self):
        return len(self.shape)

    def stride(self):
        return self.strides


def page_map(**changes):
    i32, i64 = "int32", "int64"
    a = dict(page_size=16, lengths=T(i32, 5), new_tokens=T(i32, 5), pool=T(i32, 40), cursor=T(i64, 2), table=T(i32, 5, 8), lengths_after=T(i32, 5),
             row_start=T(i32, 6), slots=T(i64, 9), positions=T(i32, 9), request=T(i32, 9), cursor_after=T(i64, 2), unplaced=T(i64, 1))
    return fc.PageMap(**{**a, **changes})


def heads(grad=False, dtype="bfloat16", dim=64, tokens=7, **changes):
    a = dict(q=T(dtype, tokens, 4, dim), k=T(dtype, tokens, 2, dim), q_weight=T(dtype, dim), k_weight=T(dtype, dim), cos_sin=T("float32", 100, dim),
             positions=T("int32", 1, tokens))
    if grad:
        a |= dict(dq_out=T(dtype, tokens, 4, dim), dk_out=T(dtype, tokens, 2, dim), dq=T(dtype, tokens, 4, dim), dk=T(dtype, tokens, 2, dim),
                  dq_weight=T("float32", dim), dk_weight=T("float32", dim))
    else:
        a |= dict(q_out=T(dtype, tokens, 4, dim), k_out=T(dtype, tokens, 2, dim))
    return (fc.HeadNormRopeGrad if grad else fc.HeadNormRope)(**{**a, **changes})


def into_cache(dtype="bfloat16", **changes):
    return heads(**{**dict(dtype=dtype, k_out=None, v=T(dtype, 7, 2, 64), k_cache=T(dtype, 9, 16, 2, 64), v_cache=T(dtype, 9, 16, 2, 64), slots=T("int64", 7)),
                    **changes})


def attention(dtype="bfloat16", dim=64, hq=4, hk=2, **changes):
    a = dict(q=T(dtype, 3, hq, dim), k_cache=T(dtype, 9, 16, hk, dim), v_cache=T(dtype, 9, 16, hk, dim), table=T("int32", 3, 8), lengths=T("int32", 3),
             out=T(dtype, 3, hq, dim), lse=T("float32", 3, hq))
    return fc.PagedAttention(**{**a, **changes})


ACCEPTED = [
    page_map(), page_map(table=T("int32", 5, 8, stride=(11, 1))), page_map(slots=T("int64", 0), positions=T("int32", 0), request=T("int32", 0, ptr=0)),
    page_map(lengths=T("int32", 1), new_tokens=T("int32", 1), table=T("int32", 1, 1, stride=(7, 7)), lengths_after=T("int32", 1), row_start=T("int32", 2)),
    heads(), heads(dtype="float32"), heads(dtype="float16", interleaved=True), heads(q_weight=None, k_weight=None), heads(cos_sin=None, positions=None),
    heads(dim=512), heads(dim=2), heads(tokens=0), heads(eps=0.0), heads(axis_of=T("int32", 32), positions=T("int32", 3, 7)),
    heads(q=T("bfloat16", 7, 4, 64, stride=(0, 64, 1))), heads(q=T("bfloat16", 7, 4, 64, ptr=0x20000002)),
    into_cache(), into_cache(k_cache=T("bfloat16", 9, 16, 2, 64, stride=(2048, 64, 1024, 1))), into_cache(dtype="float32"),
    heads(True), heads(True, q_weight=None, dq_weight=None), heads(True, tokens=0),
    attention(), attention(dtype="float32"), attention(dtype="float16", dim=256), attention(dim=8), attention(hq=7, hk=1), attention(lse=None),
    attention(window=5), attention(scale=-1.0), attention(k_cache=T("bfloat16", 9, 16, 2, 64, stride=(2048, 64, 1024, 1))),
    attention(table=T("int32", 3, 0), k_cache=T("bfloat16", 0, 16, 2, 64, ptr=0), v_cache=T("bfloat16", 0, 16, 2, 64, ptr=0)),
]

REFUSED = [
    # wrong shapes, types, strides, sizes
    ("FC_E_ARG", lambda: page_map(page_size=0)),
    ("FC_E_ARG", lambda: page_map(new_tokens=T("int32", 4))),
    ("FC_E_ARG", lambda: page_map(new_tokens=T("int64", 5))),
    ("FC_E_ARG", lambda: page_map(row_start=T("int32", 5))),
    ("FC_E_ARG", lambda: page_map(positions=T("int32", 8))),
    ("FC_E_ARG", lambda: page_map(slots=T("int32", 9))),
    ("FC_E_ARG", lambda: page_map(cursor=T("int64", 3))),
    ("FC_E_ARG", lambda: page_map(table=T("int32", 5, 8, stride=(4, 1)))),
    ("FC_E_ARG", lambda: page_map(table=T("int32", 5, 8, stride=(1, 5)))),
    ("FC_E_ARG", lambda: page_map(lengths=None)),
    ("FC_E_LIMIT", lambda: page_map(table=T("int32", 5, 1 << 30))),
    ("FC_E_LIMIT", lambda: page_map(pool=T("int32", 1 << 31))),
    ("FC_E_UNBOUND", lambda: page_map(pool=T("int32", 40, ptr=0))),
    ("FC_E_UNBOUND", lambda: page_map(cursor=T("int64", 2, ptr=0x20000004))),
    ("FC_E_ARG", lambda: heads(dtype="int32")),
    ("FC_E_ARG", lambda: heads(k=T("float16", 7, 2, 64))),
    ("FC_E_ARG", lambda: heads(k=T("bfloat16", 6, 2, 64))),
    ("FC_E_ARG", lambda: heads(k=T("bfloat16", 7, 2, 32))),
    ("FC_E_ARG", lambda: heads(q_weight=T("bfloat16", 32))),
    ("FC_E_ARG", lambda: heads(q_weight=T("float32", 64))),
    ("FC_E_ARG", lambda: heads(cos_sin=T("float32", 100, 63))),
    ("FC_E_ARG", lambda: heads(cos_sin=T("float32", 100, 66))),
    ("FC_E_ARG", lambda: heads(cos_sin=T("bfloat16", 100, 64))),
    ("FC_E_ARG", lambda: heads(positions=None)),
    ("FC_E_ARG", lambda: heads(cos_sin=None)),
    ("FC_E_ARG", lambda: heads(positions=T("int32", 1, 8))),
    ("FC_E_ARG", lambda: heads(axis_of=T("int32", 31))),
    ("FC_E_ARG", lambda: heads(eps=-1.0)),
    ("FC_E_ARG", lambda: heads(eps=math.nan)),
    ("FC_E_ARG", lambda: heads(eps=1e39)),                                                 # infinite in 32 bits
    ("FC_E_ARG", lambda: heads(True, eps=math.inf)),
    ("FC_E_ARG", lambda: heads(q_out=T("bfloat16", 7, 4, 64, stride=(0, 64, 1)))),
    ("FC_E_ARG", lambda: heads(q_out=T("bfloat16", 7, 4, 64, stride=(256, 64, 2)))),
    ("FC_E_ARG", lambda: heads(q_out=T("bfloat16", 7, 5, 64))),
    ("FC_E_ARG", lambda: heads(q=T("bfloat16", 7, 4, 64, stride=(-256, 64, 1)))),
    ("FC_E_ARG", lambda: heads(v=T("bfloat16", 7, 2, 64))),
    ("FC_E_ARG", lambda: heads(k_out=None)),
    ("FC_E_UNSUPPORTED", lambda: heads(dim=514)),
    ("FC_E_UNSUPPORTED", lambda: heads(dim=63, cos_sin=None, positions=None)),
    ("FC_E_UNSUPPORTED", lambda: heads(dim=256, cos_sin=T("float32", 100, 250))),
    ("FC_E_UNBOUND", lambda: heads(q=T("bfloat16", 7, 4, 64, ptr=0x20000001))),
    ("FC_E_LIMIT", lambda: heads(q=T("bfloat16", 7, 4, 64, stride=(1 << 43, 64, 1)))),
    ("FC_E_ARG", lambda: into_cache(k_out=T("bfloat16", 7, 2, 64))),
    ("FC_E_ARG", lambda: into_cache(slots=T("int32", 7))),
    ("FC_E_ARG", lambda: into_cache(v=None)),
    ("FC_E_ARG", lambda: into_cache(v_cache=T("bfloat16", 9, 16, 3, 64))),
    ("FC_E_ARG", lambda: into_cache(v_cache=T("bfloat16", 9, 8, 2, 64))),
    ("FC_E_ARG", lambda: into_cache(k_cache=T("bfloat16", 9, 16, 2, 64, stride=(0, 128, 64, 1)))),
    ("FC_E_ARG", lambda: into_cache(k_cache=T("bfloat16", 9, 0, 2, 64), v_cache=T("bfloat16", 9, 0, 2, 64))),
    ("FC_E_ARG", lambda: heads(True, dk=T("bfloat16", 7, 3, 64))),
    ("FC_E_ARG", lambda: heads(True, dq_weight=T("bfloat16", 64))),
    ("FC_E_ARG", lambda: heads(True, dq_weight=None)),
    ("FC_E_ARG", lambda: heads(True, k_weight=None)),
    ("FC_E_ARG", lambda: attention(dtype="int32")),
    ("FC_E_ARG", lambda: attention(hq=5)),
    ("FC_E_ARG", lambda: attention(hk=0)),
    ("FC_E_ARG", lambda: attention(v_cache=T("bfloat16", 9, 16, 2, 32))),
    ("FC_E_ARG", lambda: attention(k_cache=T("float16", 9, 16, 2, 64))),
    ("FC_E_ARG", lambda: attention(table=T("int32", 2, 8))),
    ("FC_E_ARG", lambda: attention(table=T("int64", 3, 8))),
    ("FC_E_ARG", lambda: attention(lengths=T("int32", 4))),
    ("FC_E_ARG", lambda: attention(out=T("float32", 3, 4, 64))),
    ("FC_E_ARG", lambda: attention(out=T("bfloat16", 3, 4, 64, stride=(0, 64, 1)))),
    ("FC_E_ARG", lambda: attention(lse=T("bfloat16", 3, 4))),
    ("FC_E_ARG", lambda: attention(window=-1)),
    ("FC_E_ARG", lambda: attention(scale=math.inf)),
    ("FC_E_ARG", lambda: attention(scale=math.nan)),
    ("FC_E_ARG", lambda: attention(scale=-1e39)),
    ("FC_E_ARG", lambda: attention(k_cache=T("bfloat16", 9, 0, 2, 64), v_cache=T("bfloat16", 9, 0, 2, 64))),
    ("FC_E_UNSUPPORTED", lambda: attention(dim=264)),
    ("FC_E_UNSUPPORTED", lambda: attention(dim=60)),
    ("FC_E_UNBOUND", lambda: attention(k_cache=T("bfloat16", 9, 16, 2, 64, ptr=0x20000008))),
    ("FC_E_UNBOUND", lambda: attention(q=T("bfloat16", 3, 4, 64, ptr=0x20000008))),
    ("FC_E_UNBOUND", lambda: attention(v_cache=T("bfloat16", 9, 16, 2, 64, stride=(2052, 128, 64, 1)))),
    ("FC_E_UNBOUND", lambda: attention(table=T("int32", 3, 8, ptr=0))),
]


@pytest.mark.parametrize("k", range(len(ACCEPTED)))
def test_operators_that_are_right_are_bound(k):
    assert fc.fc_operators_scratch_bytes([ACCEPTED[k]]) >= B.FC_SCRATCH_CONTROL_BYTES
    fc.BoundOperators([ACCEPTED[k]], SCRATCH)


@pytest.mark.parametrize("k", range(len(REFUSED)))
def test_operators_that_are_wrong_are_refused(k):
    code, make = REFUSED[k]
    op = make()
    for call in (lambda: fc.fc_operators_scratch_bytes([page_map(), op]), lambda: fc.fc_run_operators([page_map(), op], SCRATCH),
                 lambda: fc.BoundOperators([page_map(), op], SCRATCH)):
        with pytest.raises(fc.FcError) as e:
            call()
        assert e.value.name == code and "operator 1: " in str(e.value), str(e.value)


def test_lists_and_scratch_that_are_wrong_are_refused():
    def expect(code, f):
        with pytest.raises(fc.FcError) as e:
            f()
        assert e.value.name == code, str(e.value)
    need = fc.fc_operators_scratch_bytes([attention(), heads(True)])
    assert need == max(fc.fc_operators_scratch_bytes([op]) for op in (attention(), heads(True)))       # they run one after the other
    expect("FC_E_SCRATCH", lambda: fc.fc_run_operators([attention(), heads(True)], (0x10000000, need - 1)))
    expect("FC_E_SCRATCH", lambda: fc.fc_run_operators([page_map()], (0, 1 << 30)))
    expect("FC_E_SCRATCH", lambda: fc.fc_run_operators([page_map()], (0x10000010, 1 << 30)))
    lib = B.lib()
    ops = B._operators([page_map()])
    assert lib.fc_run_operators(None, 1, SCRATCH[0], SCRATCH[1], None) == -7
    assert lib.fc_run_operators(ops, -1, SCRATCH[0], SCRATCH[1], None) == -7
    assert lib.fc_operators_scratch_bytes(ops, 1, None) == -7
    assert lib.fc_bind_operators(ops, 1, SCRATCH[0], SCRATCH[1], None) == -7
    ops[0].kind = 17
    assert lib.fc_run_operators(ops, 1, SCRATCH[0], SCRATCH[1], None) == -7 and "unknown kind 17" in fc.fc_last_error()
    ops[0].kind, ops[0].args = 0, None
    assert lib.fc_run_operators(ops, 1, SCRATCH[0], SCRATCH[1], None) == -7
    fc.fc_run_operators([], SCRATCH)
    fc.fc_run_operators([attention(q=T("bfloat16", 0, 4, 64), table=T("int32", 0, 8), lengths=T("int32", 0), out=T("bfloat16", 0, 4, 64), lse=None)], SCRATCH)


def test_tensors_the_binding_does_not_take():
    import torch
    for bad in (torch.zeros(5, dtype=torch.int32), T("float64", 5), T("int32"), T("int32", 1, 1, 1, 1, 5)):
        with pytest.raises(ValueError):
            page_map(lengths=bad)


def test_a_copy_of_bound_operators_shares_them():
    import copy
    bound = fc.BoundOperators([attention()], SCRATCH)
    other = copy.copy(bound)
    assert other._handle is bound._handle
    with pytest.raises((TypeError, ValueError)):
        copy.deepcopy(bound)


def test_struct_layout_matches_the_binding(tmp_path):
    names = ["fc_tensor", "fc_operator", "fc_page_map", "fc_head_norm_rope", "fc_head_norm_rope_grad", "fc_paged_attention"]
    fields = [(n, f) for n in names for f, _ in getattr(B, n)._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "fc.h"\nint main(void){'
                   + "".join(f'printf("%zu\\n", sizeof({n}));' for n in names) + "".join(f'printf("%zu\\n", offsetof({n}, {f}));' for n, f in fields)
                   + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(getattr(B, n)) for n in names] + [getattr(getattr(B, n), f).offset for n, f in fields]


# --------------------------------------------------------------------------- the oracle
def test_oracle_of_the_page_map_by_hand():
    # pages of 4; request 0 grows within its page, 1 is new and takes two pages, 2 leaves and gives back two, 3 gets none of the one it needs
    got = O.page_map(4, [2, 0, 7, 4], [1, 6, -7, 1], np.array([50, 51, 52, 53, 54], np.int32), [7, 9],
                     np.array([[10, 0, 0], [0, 0, 0], [20, 21, 0], [30, 0, 0]], np.int32), 10)
    assert got["table"].tolist() == [[10, 0, 0], [52, 53, 0], [20, 21, 0], [30, 0, 0]]
    assert got["pool"].tolist() == [21, 51, 52, 53, 20]
    assert got["lengths_after"].tolist() == [3, 6, 0, 4] and got["row_start"].tolist() == [0, 1, 7, 7, 8]
    assert got["slots"].tolist() == [42, 208, 209, 210, 211, 212, 213, -1, -1, -1]
    assert got["positions"].tolist() == [2, 0, 1, 2, 3, 4, 5, 4, 0, 0] and got["request"].tolist() == [0, 1, 1, 1, 1, 1, 1, 3, -1, -1]
    assert got["cursor_after"].tolist() == [9, 11] and got["unplaced"].tolist() == [1]


@pytest.mark.parametrize("interleaved", [False, True])
def test_oracle_of_the_rotation_as_complex_numbers_and_as_a_rotation(interleaved):
    rng = np.random.default_rng(1)
    x, angle = rng.standard_normal((5, 3, 12)), rng.uniform(-3, 3, (9, 4))
    table, positions = np.concatenate([np.cos(angle), np.sin(angle)], 1), rng.integers(0, 9, (2, 5)).astype(np.int32)
    c, s = O.angles(table, positions, np.array([0, 1, 1, 0]))
    got = O.head_norm_rope(x, None, 0.0, c, s, interleaved)
    a, b = (x[..., 0:8:2], x[..., 1:8:2]) if interleaved else (x[..., :4], x[..., 4:8])
    turn = np.stack([np.exp(1j * angle[positions[k], i]) for i, k in enumerate([0, 1, 1, 0])], 1)
    z = (a + 1j * b) * turn[:, None, :]
    want = x.copy()
    want[..., 0:8:2 if interleaved else 1][..., :4], want[..., (1 if interleaved else 4):8:2 if interleaved else 1] = z.real, z.imag
    assert np.allclose(got, want, atol=1e-14) and np.array_equal(got[..., 8:], x[..., 8:])
    assert np.allclose((got ** 2).sum(-1), (x ** 2).sum(-1))
    assert np.allclose(O.turned(got, c, -s, interleaved), x)
    far = O.angles(table, np.full((1, 5), 9, np.int32), None)
    assert np.isnan(far[0]).all() and np.isnan(far[1]).all()


def test_oracle_of_the_norm_and_its_gradient():
    rng = np.random.default_rng(2)
    x, w, dy = rng.standard_normal((4, 3, 10)), rng.uniform(0.5, 2, 10), rng.standard_normal((4, 3, 10))
    y = O.head_norm_rope(x, np.ones(10), 0.0, None, None, False)
    assert np.allclose((y ** 2).mean(-1), 1)
    angle = rng.uniform(-3, 3, (4, 4))
    c, s = np.cos(angle), np.sin(angle)
    dx, dw = O.head_norm_rope_grad(x, w, 1e-3, c, s, True, dy)
    value = lambda x, w: (O.head_norm_rope(x, w, 1e-3, c, s, True) * dy).sum()  # noqa: E731
    for at in np.ndindex(2, 2, 10):
        step = np.zeros_like(x)
        step[at] = 1e-6
        assert abs((value(x + step, w) - value(x - step, w)) / 2e-6 - dx[at]) < 1e-7
    for d in range(10):
        step = np.zeros(10)
        step[d] = 1e-6
        assert abs((value(x, w + step) - value(x, w - step)) / 2e-6 - dw[d]) < 1e-6


def test_oracle_of_attention_against_closed_forms():
    rng = np.random.default_rng(3)
    k, v, q = rng.standard_normal((6, 4, 2, 8)), rng.standard_normal((6, 4, 2, 8)), rng.standard_normal((3, 4, 8))
    table = np.array([[3, 1, -1], [5, 9, 0], [2, 4, 0]])
    out, lse, _, _ = O.paged_attention(q, k, v, table, [5, 10, 0], 0.0)                  # all weights equal: means, and log of the number of keys
    rows = np.concatenate([v[3], v[1, :1]])
    assert np.allclose(out[0], rows.mean(0)[[0, 0, 1, 1]]) and np.allclose(lse[0], np.log(5))
    rows = np.concatenate([v[5], v[0, :2]])                                              # page 9 is not there
    assert np.allclose(out[1], rows.mean(0)[[0, 0, 1, 1]]) and np.allclose(lse[1], np.log(6))
    assert (out[2] == 0).all() and (lse[2] == -np.inf).all()
    out, lse, _, _ = O.paged_attention(q, k, v, table, [5, 10, 3], 0.5, window=1)        # one key: its value, and its score
    assert np.allclose(out[2], v[2, 2][[0, 0, 1, 1]]) and np.allclose(lse[2], 0.5 * (q[2] * k[2, 2][[0, 0, 1, 1]]).sum(-1))
