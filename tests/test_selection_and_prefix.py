"""Bounds of pages, the selection of pages by them, attention over a table for each key head and over shared prefixes: what is taken and refused
before anything is enqueued, the structs of the ABI, and the oracle against closed forms.  No GPU: the arrays are addresses that nothing reads."""
import ctypes
import math
import os
import subprocess

import numpy as np
import pytest

import paper_2407_13585_amd as fc
from oracle import cache as O
from paper_2407_13585_amd import binding as B
from test_operator_limits import expect, taken
from test_operators import SCRATCH, T, attention, page_map

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def bounds(dtype="bfloat16", dim=64, **changes):
    a = dict(k_cache=T(dtype, 9, 16, 2, dim), table=T("int32", 3, 8), lengths_before=T("int32", 3), lengths=T("int32", 3), bounds=T(dtype, 9, 2, 2, dim))
    return fc.PageBounds(**{**a, **changes})


def select(dtype="bfloat16", dim=64, hq=4, hk=2, **changes):
    a = dict(q=T(dtype, 3, hq, dim), bounds=T(dtype, 9, hk, 2, dim), table=T("int32", 3, 8), lengths=T("int32", 3), page_size=16,
             selected=T("int32", 3, hk, 5), selected_lengths=T("int32", 3, hk))
    return fc.PageSelect(**{**a, **changes})


def of_heads(**changes):
    return attention(**{**dict(table=T("int32", 3, 2, 8), lengths=T("int32", 3, 2)), **changes})


def prefix(dtype="bfloat16", dim=64, hq=4, hk=2, **changes):
    a = dict(q=T(dtype, 3, hq, dim), k_cache=T(dtype, 9, 16, hk, dim), v_cache=T(dtype, 9, 16, hk, dim), prefix_table=T("int32", 2, 6),
             prefix_lengths=T("int32", 2), group_start=T("int32", 3), table=T("int32", 3, 8), lengths=T("int32", 3), out=T(dtype, 3, hq, dim),
             lse=T("float32", 3, hq))
    return fc.PrefixAttention(**{**a, **changes})


ACCEPTED = [
    bounds(), bounds(dtype="float32"), bounds(dtype="float16", dim=256), bounds(dim=8), bounds(table=T("int32", 3, 0)), bounds(table=T("int32", 3, 8, stride=(11, 1))),
    bounds(k_cache=T("bfloat16", 9, 16, 2, 64, stride=(2048, 64, 1024, 1))), bounds(bounds=T("bfloat16", 9, 2, 2, 64, stride=(512, 72, 200, 1))),
    bounds(k_cache=T("bfloat16", 0, 16, 2, 64, ptr=0), bounds=T("bfloat16", 0, 2, 2, 64, ptr=0)),
    bounds(table=T("int32", 0, 8, ptr=0), lengths_before=T("int32", 0), lengths=T("int32", 0)),
    select(), select(dtype="float32"), select(dtype="float16", dim=256), select(dim=8), select(hq=17, hk=1), select(first=0, last=0), select(first=2, last=3),
    select(selected=T("int32", 3, 2, 0), first=0, last=0), select(table=T("int32", 3, 0)), select(q=T("bfloat16", 3, 4, 64, stride=(0, 64, 1))),
    select(selected=T("int32", 3, 2, 5, stride=(5, 20, 1)), selected_lengths=T("int32", 3, 2, stride=(7, 1))), select(page_size=(1 << 31) // 5),
    of_heads(), of_heads(dtype="float32"), of_heads(window=3), of_heads(lengths=T("int32", 3, 2, stride=(9, 1)), table=T("int32", 3, 2, 8, stride=(8, 40, 1))),
    of_heads(table=T("int32", 3, 2, 0)), of_heads(lse=None),
    prefix(), prefix(dtype="float32"), prefix(dtype="float16", dim=256), prefix(dim=8), prefix(hq=34), prefix(lse=None), prefix(scale=-1.0), prefix(scale=0.0),
    prefix(prefix_table=T("int32", 0, 6, ptr=0), prefix_lengths=T("int32", 0, ptr=0), group_start=T("int32", 1)),
    prefix(prefix_table=T("int32", 2, 0, ptr=0)), prefix(prefix_table=T("int32", 1024, 6), prefix_lengths=T("int32", 1024), group_start=T("int32", 1025)),
    prefix(k_cache=T("bfloat16", 0, 16, 2, 64, ptr=0), v_cache=T("bfloat16", 0, 16, 2, 64, ptr=0)),
    prefix(q=T("bfloat16", 0, 4, 64), table=T("int32", 0, 8), lengths=T("int32", 0), out=T("bfloat16", 0, 4, 64), lse=None),
]

REFUSED = [
    ("FC_E_ARG", lambda: bounds(dtype="int32")),
    ("FC_E_ARG", lambda: bounds(k_cache=T("float16", 9, 16, 2, 64))),
    ("FC_E_ARG", lambda: bounds(bounds=T("bfloat16", 9, 2, 64))),
    ("FC_E_ARG", lambda: bounds(bounds=T("bfloat16", 8, 2, 2, 64))),
    ("FC_E_ARG", lambda: bounds(bounds=T("bfloat16", 9, 2, 1, 64))),
    ("FC_E_ARG", lambda: bounds(bounds=T("bfloat16", 9, 2, 2, 64, stride=(256, 128, 0, 1)))),
    ("FC_E_ARG", lambda: bounds(bounds=T("bfloat16", 9, 2, 2, 64, stride=(256, 64, 64, 1)))),
    ("FC_E_ARG", lambda: bounds(table=T("int64", 3, 8))),
    ("FC_E_ARG", lambda: bounds(lengths=T("int32", 2))),
    ("FC_E_ARG", lambda: bounds(lengths_before=T("int32", 4))),
    ("FC_E_ARG", lambda: bounds(lengths_before=None)),
    ("FC_E_ARG", lambda: bounds(k_cache=T("bfloat16", 9, 0, 2, 64))),
    ("FC_E_UNSUPPORTED", lambda: bounds(dim=264)),
    ("FC_E_UNSUPPORTED", lambda: bounds(dim=60)),
    ("FC_E_UNBOUND", lambda: bounds(k_cache=T("bfloat16", 9, 16, 2, 64, ptr=0x20000008))),
    ("FC_E_UNBOUND", lambda: bounds(bounds=T("bfloat16", 9, 2, 2, 64, stride=(260, 128, 64, 1)))),
    ("FC_E_UNBOUND", lambda: bounds(bounds=T("bfloat16", 9, 2, 2, 64, ptr=0))),
    ("FC_E_ARG", lambda: select(dtype="int32")),
    ("FC_E_ARG", lambda: select(hq=5)),
    ("FC_E_ARG", lambda: select(hk=0)),
    ("FC_E_ARG", lambda: select(hq=0)),
    ("FC_E_ARG", lambda: select(bounds=T("float32", 9, 2, 2, 64))),
    ("FC_E_ARG", lambda: select(bounds=T("bfloat16", 9, 2, 2, 32))),
    ("FC_E_ARG", lambda: select(table=T("int32", 2, 8))),
    ("FC_E_ARG", lambda: select(lengths=T("int32", 3, 1))),
    ("FC_E_ARG", lambda: select(selected=T("int64", 3, 2, 5))),
    ("FC_E_ARG", lambda: select(selected=T("int32", 3, 4, 5))),
    ("FC_E_ARG", lambda: select(selected=T("int32", 3, 2, 5, stride=(5, 5, 1)))),
    ("FC_E_ARG", lambda: select(selected_lengths=T("int32", 3))),
    ("FC_E_ARG", lambda: select(page_size=0)),
    ("FC_E_ARG", lambda: select(first=-1)),
    ("FC_E_ARG", lambda: select(last=-1)),
    ("FC_E_ARG", lambda: select(first=3, last=3)),
    ("FC_E_ARG", lambda: select(first=(1 << 31) - 1, last=(1 << 31) - 1)),
    ("FC_E_ARG", lambda: select(selected=T("int32", 3, 2, 0))),
    ("FC_E_LIMIT", lambda: select(page_size=(1 << 31) // 5 + 1)),
    ("FC_E_UNSUPPORTED", lambda: select(dim=264)),
    ("FC_E_UNSUPPORTED", lambda: select(dim=4)),
    ("FC_E_UNBOUND", lambda: select(q=T("bfloat16", 3, 4, 64, ptr=0x20000008))),
    ("FC_E_UNBOUND", lambda: select(bounds=T("bfloat16", 9, 2, 2, 64, stride=(256, 128, 68, 1)))),
    ("FC_E_UNBOUND", lambda: select(selected=T("int32", 3, 2, 5, ptr=0))),
    ("FC_E_ARG", lambda: of_heads(table=T("int32", 3, 4, 8))),
    ("FC_E_ARG", lambda: of_heads(lengths=T("int32", 3))),
    ("FC_E_ARG", lambda: of_heads(table=T("int32", 3, 8))),
    ("FC_E_ARG", lambda: of_heads(lengths=T("int32", 3, 4))),
    ("FC_E_ARG", lambda: of_heads(window=-1)),
    ("FC_E_ARG", lambda: prefix(dtype="int32")),
    ("FC_E_ARG", lambda: prefix(hq=5)),
    ("FC_E_ARG", lambda: prefix(hk=0)),
    ("FC_E_ARG", lambda: prefix(prefix_table=T("int32", 2))),
    ("FC_E_ARG", lambda: prefix(prefix_lengths=T("int32", 3))),
    ("FC_E_ARG", lambda: prefix(group_start=T("int32", 2))),
    ("FC_E_ARG", lambda: prefix(group_start=T("int64", 3))),
    ("FC_E_ARG", lambda: prefix(group_start=None)),
    ("FC_E_ARG", lambda: prefix(table=T("int32", 3, 2, 8))),
    ("FC_E_ARG", lambda: prefix(lengths=T("int32", 2))),
    ("FC_E_ARG", lambda: prefix(v_cache=T("bfloat16", 9, 16, 2, 32))),
    ("FC_E_ARG", lambda: prefix(out=T("bfloat16", 3, 4, 64, stride=(0, 64, 1)))),
    ("FC_E_ARG", lambda: prefix(lse=T("bfloat16", 3, 4))),
    ("FC_E_ARG", lambda: prefix(scale=math.nan)),
    ("FC_E_ARG", lambda: prefix(scale=1e39)),
    ("FC_E_UNSUPPORTED", lambda: prefix(scale=-1e38)),
    ("FC_E_ARG", lambda: prefix(k_cache=T("bfloat16", 9, 0, 2, 64), v_cache=T("bfloat16", 9, 0, 2, 64))),
    ("FC_E_UNSUPPORTED", lambda: prefix(dim=264)),
    ("FC_E_UNSUPPORTED", lambda: prefix(dim=60)),
    ("FC_E_UNBOUND", lambda: prefix(q=T("bfloat16", 3, 4, 64, ptr=0x20000008))),
    ("FC_E_UNBOUND", lambda: prefix(prefix_table=T("int32", 2, 6, ptr=0))),
    ("FC_E_LIMIT", lambda: prefix(prefix_table=T("int32", 1025, 6), prefix_lengths=T("int32", 1025), group_start=T("int32", 1026))),
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


def test_numbers_that_the_abi_would_cut_short_are_refused():
    for make in (lambda: select(page_size=1 << 31), lambda: select(first=1 << 32), lambda: select(last=-(1 << 31) - 1)):
        with pytest.raises(ValueError):
            make()


# --------------------------------------------------------------------------- extents that cannot be counted
def test_bounds_count_requests_pages_and_heads_in_full():
    def of(requests, width, hk=1, page=16):
        return bounds(k_cache=T("bfloat16", 9, page, hk, 64), bounds=T("bfloat16", 9, hk, 2, 64), table=T("int32", requests, width, stride=(0, 1)),
                      lengths_before=T("int32", requests), lengths=T("int32", requests))
    most = (1 << 31) - 1
    expect("FC_E_LIMIT", of(1 << 16, 1 << 15))
    expect("FC_E_LIMIT", of(most, most, hk=1 << 10))
    expect("FC_E_LIMIT", of(most, 1, hk=2))
    taken(of(1 << 16, (1 << 15) - 1))
    taken(of(most, 1))
    taken(of(15, most))                                      # of which a request of 2^31-1 keys has 2^27
    expect("FC_E_LIMIT", of(16, most))


def test_selections_count_requests_heads_and_pages_in_full():
    def of(requests, hk=1, width=1):
        return select(hk=hk, hq=hk, q=T("bfloat16", requests, hk, 64, stride=(0, 64, 1)), table=T("int32", requests, width, stride=(0, 1)),
                      lengths=T("int32", requests), selected=T("int32", requests, hk, 5), selected_lengths=T("int32", requests, hk))
    expect("FC_E_LIMIT", of(1 << 24))
    expect("FC_E_LIMIT", of((1 << 31) - 1, hk=1 << 12))
    expect("FC_E_LIMIT", of(1 << 14, hk=1, width=(1 << 22) + 1))
    taken(of((1 << 24) - 1))
    fc.fc_operators_scratch_bytes([of(1 << 14, hk=1, width=1 << 22)])


def test_key_heads_with_tables_of_their_own_are_counted_in_full():
    def of(requests, hk):
        return of_heads(hk=hk, hq=hk, q=T("bfloat16", requests, hk, 64, stride=(0, 64, 1)), out=T("bfloat16", requests, hk, 64), lse=None,
                        table=T("int32", requests, hk, 0), lengths=T("int32", requests, hk))
    expect("FC_E_LIMIT", of(1 << 30, 2))
    expect("FC_E_LIMIT", of(1 << 20, 1 << 20))
    taken(of(1 << 15, 1 << 15))


def test_prefixes_count_their_keys_heads_and_groups_in_full():
    def of(width, page=65536, groups=1, requests=3, hq=4, hk=2):
        cache = T("bfloat16", 9, page, hk, 64)
        return prefix(hq=hq, hk=hk, k_cache=cache, v_cache=cache, prefix_table=T("int32", groups, width, stride=(0, 1)), prefix_lengths=T("int32", groups),
                      group_start=T("int32", groups + 1), q=T("bfloat16", requests, hq, 64, stride=(0, 64, 1)), out=T("bfloat16", requests, hq, 64), lse=None,
                      table=T("int32", requests, 1), lengths=T("int32", requests))
    for width in (1 << 22, 1 << 23, (1 << 31) - 1):          # 2^31-1 keys of a prefix are 2^24 pieces of 128
        taken(of(width, hk=1))
        expect("FC_E_LIMIT", of(width, groups=64, requests=64, hk=4))
    expect("FC_E_LIMIT", of(1 << 15, groups=1, requests=1 << 14, hq=1 << 10, hk=1))
    expect("FC_E_LIMIT", of(1, page=16, requests=1 << 30, hq=4, hk=4))


def test_struct_layout_matches_the_binding(tmp_path):
    names = ["fc_page_bounds", "fc_page_select", "fc_prefix_attention"]
    fields = [(n, f) for n in names for f, _ in getattr(B, n)._fields_]
    kinds = {"FC_PAGE_BOUNDS": fc.PageBounds.kind, "FC_PAGE_SELECT": fc.PageSelect.kind, "FC_PREFIX_ATTENTION": fc.PrefixAttention.kind}
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "fc.h"\nint main(void){'
                   + "".join(f'printf("%zu\\n", sizeof({n}));' for n in names) + "".join(f'printf("%zu\\n", offsetof({n}, {f}));' for n, f in fields)
                   + "".join(f'printf("%d\\n", (int){k});' for k in kinds) + "return 0;}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [ctypes.sizeof(getattr(B, n)) for n in names] + [getattr(getattr(B, n), f).offset for n, f in fields] + list(kinds.values())


# --------------------------------------------------------------------------- the oracle
def test_oracle_of_bounds_by_hand():
    k = np.arange(2 * 4 * 1 * 2, dtype=float).reshape(2, 4, 1, 2) * np.array([1.0, -1.0])
    before = np.full((2, 1, 2, 2), 0.0)
    got = O.page_bounds(k, np.array([[1, 0]]), [0], [5], before)
    assert np.array_equal(got[1, 0], [[8, -15], [14, -9]]) and np.array_equal(got[0, 0], [[0, -1], [0, -1]])
    got = O.page_bounds(k, np.array([[1, 0]]), [2], [4], before)                           # the page's first keys are in its bounds
    assert np.array_equal(got[1, 0], [[0, -15], [14, 0]]) and np.array_equal(got[0], before[0])


def test_oracle_of_the_selection_bounds_what_keys_score():
    rng = np.random.default_rng(1)
    k = rng.standard_normal((6, 8, 2, 16))
    bounds = O.page_bounds(k, np.arange(6)[None], [0], [48], np.zeros((6, 2, 2, 16)))
    q = rng.standard_normal((1, 6, 16))
    for h in range(2):
        s = O.page_scores(q[0, 3 * h:3 * h + 3], bounds[:, h])
        reached = np.einsum("pjd,gd->pjg", k[:, :, h], q[0, 3 * h:3 * h + 3])
        assert (s >= reached.max((1, 2))).all()
        selected, held = O.page_select(q, bounds, np.array([[5, 4, 3, 2, 1, 0]]), [45], 8, 3, 1, 1)
        rest = [p for p in np.argsort(-s) if p not in (5, 0)]
        assert list(selected[0, h]) == [5, rest[0], 0] and held[0, h] == 8 + 8 + 5
    one = np.broadcast_to(q[0, :1, None, :].transpose(1, 0, 2), (1, 1, 16))
    assert np.isclose(O.page_scores(one[0], np.stack([one[0], one[0]], 1))[0], (one ** 2).sum())      # a page of one key: its score


def test_oracle_of_selected_and_prefix_attention_against_attention():
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, 9, 8, 2, 16))
    q, table, lengths = rng.standard_normal((3, 4, 16)), rng.permutation(9).reshape(3, 3), np.array([20, 0, 24])
    want = O.paged_attention(q, k, v, table, lengths, 0.25, 11)
    got = O.selected_attention(q, k, v, np.repeat(table[:, None], 2, 1), np.repeat(lengths[:, None], 2, 1), 0.25, 11)
    assert all(np.allclose(a, b) for a, b in zip(got, want))
    # a prefix of one page of its own, and the rest
    want = O.paged_attention(q, k, v, np.concatenate([[[4], [4], [4]], table], 1), lengths + 8, 0.25)
    got = O.prefix_attention(q, k, v, np.array([[4]]), [8], [0, 3], table, lengths, 0.25)
    assert all(np.allclose(a, b) for a, b in zip(got, want))
    got = O.prefix_attention(q, k, v, np.array([[4]]), [8], [1, 2], table, lengths, 0.25)
    alone = O.paged_attention(q, k, v, table, lengths, 0.25)
    assert np.allclose(got[0][1], want[0][1]) and np.allclose(got[0][[0, 2]], alone[0][[0, 2]])
