"""What the operators of a serving cache refuse before anything is enqueued: extents that their kernels cannot count, outputs that lie over
their inputs otherwise than they do; and what lies just beside it is taken.  No GPU: the arrays are addresses that nothing reads."""
import pytest

import paper_2407_13585_amd as fc
from paper_2407_13585_amd import binding as B
from test_operators import SCRATCH, T, attention, heads, into_cache, page_map
from workloads import Graph


def expect(code, *ops):
    for call in (lambda: fc.fc_operators_scratch_bytes(ops), lambda: fc.fc_run_operators(ops, SCRATCH), lambda: fc.BoundOperators(ops, SCRATCH)):
        with pytest.raises(fc.FcError) as e:
            call()
        assert e.value.name == code, str(e.value)


def taken(*ops):
    fc.fc_operators_scratch_bytes(ops)
    fc.BoundOperators(ops, SCRATCH)


def attention_over(width, page, requests, kv=2, group=2, dtype="bfloat16"):
    cache = T(dtype, 9, page, kv, 64)
    return attention(q=T(dtype, requests, kv * group, 64), out=T(dtype, requests, kv * group, 64), lse=None, lengths=T("int32", requests),
                     table=T("int32", requests, width, stride=(0, 1)), k_cache=cache, v_cache=cache)


@pytest.mark.parametrize("width", [1 << 22, 1 << 23, (1 << 23) + 1, 1 << 24, (1 << 31) - 1])
def test_attention_counts_the_keys_of_wide_tables_in_full(width):
    # 2^22 pages of 65536 places are 2^38 places, 2^23 are 2^32 pieces of 128: a request has up to 2^31-1 keys of them, 2^24 pieces
    expect("FC_E_LIMIT", attention_over(width, 65536, requests=300))
    expect("FC_E_LIMIT", attention_over(width, 65536, requests=64, kv=2))
    taken(attention_over(width, 65536, requests=63, kv=2))


def test_attention_counts_requests_and_heads_in_full():
    expect("FC_E_LIMIT", attention_over(0, 16, requests=1 << 30, kv=2))                   # 2^31
    expect("FC_E_LIMIT", attention_over((1 << 31) - 1, (1 << 31) - 1, requests=1 << 20, kv=1 << 20))     # 2^64
    expect("FC_E_LIMIT", attention_over(8, 16, requests=1 << 16, kv=1 << 16))             # 2^33
    taken(attention_over(0, 16, requests=(1 << 30) - 1, kv=2))
    taken(attention_over(8, 16, requests=1 << 15, kv=1 << 14))


@pytest.mark.parametrize("grad", [False, True])
def test_heads_of_a_token_are_counted_in_full(grad):
    def of(hq, hk):
        q, k = (T("bfloat16", 1, h, 2) for h in (hq, hk))
        outs = dict(dq_out=q, dk_out=k, dq=q, dk=k, dq_weight=None, dk_weight=None) if grad else dict(q_out=q, k_out=k)
        return heads(grad, dim=2, tokens=1, q=q, k=k, q_weight=None, k_weight=None, **outs)
    most = (1 << 31) - 1
    for hq, hk in ((most, most), (1 << 30, 1 << 30), (most, 1), (1, most)):
        expect("FC_E_LIMIT", of(hq, hk))
    for hq, hk in ((most, 0), (most - 1, 1), (1, most - 1)):
        taken(of(hq, hk))


def test_heads_that_go_into_the_cache_are_counted_in_full():
    def of(hq, hk):
        none = T("bfloat16", 0, 16, hk, 2, ptr=0)
        q, k = (T("bfloat16", 1, h, 2) for h in (hq, hk))
        return into_cache(q=q, k=k, v=k, q_out=q, q_weight=None, k_weight=None, cos_sin=None, positions=None, k_cache=none, v_cache=none, slots=T("int64", 1))
    expect("FC_E_LIMIT", of(2, (1 << 30) - 1))
    expect("FC_E_LIMIT", of((1 << 31) - 1, (1 << 31) - 1))
    taken(of(1, (1 << 30) - 1))


def test_attention_counts_the_elements_of_a_request_in_full():
    def of(heads, dim):
        cache, row = T("bfloat16", 9, 16, 1, dim), T("bfloat16", 1, heads, dim)
        return attention(q=row, out=row, lse=None, lengths=T("int32", 1), table=T("int32", 1, 8), k_cache=cache, v_cache=cache)
    for heads_, dim in ((1 << 26, 256), ((1 << 31) - 1, 8), (1 << 30, 8), (1 << 25, 256)):
        expect("FC_E_LIMIT", of(heads_, dim))
    for heads_, dim in (((1 << 25) - 1, 256), ((1 << 30) - 1, 8)):
        taken(of(heads_, dim))


def test_outputs_in_place_lie_as_their_inputs_do():
    def lying(heads_, stride, ptr=0x20000000):
        return T("bfloat16", 7, heads_, 64, stride=stride, ptr=ptr)
    # the heads' rows of one projection in place, and rows of a single head, whose stride between heads means nothing
    taken(heads(q=lying(4, (512, 64, 1)), q_out=lying(4, (512, 64, 1))))
    taken(heads(q=lying(1, (64, 999, 1)), q_out=lying(1, (64, 64, 1)), k=lying(1, (64, 5, 1)), k_out=lying(1, (64, 64, 1))))
    taken(heads(q_out=lying(4, (64, 448, 1), ptr=0x30000000)))
    taken(heads(tokens=0, q_out=T("bfloat16", 0, 4, 64, stride=(64, 448, 1))))
    # the same address, transposed or with gaps
    for stride in ((64, 448, 1), (512, 64, 1)):
        expect("FC_E_ARG", heads(q_out=lying(4, stride)))
        expect("FC_E_ARG", heads(q=lying(4, stride)))
        expect("FC_E_ARG", into_cache(q_out=lying(4, stride)))
        expect("FC_E_ARG", heads(True, dq=lying(4, stride)))
        expect("FC_E_ARG", heads(k_out=lying(2, stride)))
        expect("FC_E_ARG", heads(True, dk_out=lying(2, stride)))


def test_numbers_that_the_abi_would_cut_short_are_refused():
    for make in (lambda n: attention(window=n), lambda n: page_map(page_size=n)):
        for n in (1 << 31, (1 << 32) + 16, 1 << 64, -(1 << 31) - 1):
            with pytest.raises(ValueError, match="32 bits"):
                make(n)
        taken(make((1 << 31) - 1))
    with pytest.raises(TypeError):
        attention(window=16.0)


@pytest.mark.parametrize("grad", [False, True])
def test_an_eps_that_32_bits_take_for_zero_is_refused(grad):
    # 2^-149 is the smallest number of 32 bits, half of it is rounded to 0: a row of zeros would be NaN, not zeros
    for eps in (2.0 ** -150, 1e-46, 1e-300):
        expect("FC_E_ARG", heads(grad, eps=eps))
    for eps in (0.0, 2.0 ** -149, 1e-38):
        taken(heads(grad, eps=eps))


def spmv_of_many_rows(rows, elements, cols=1500000):
    g = Graph()
    g.add("x", "input", "f32", (cols,))
    g.add("col", "input", "i32", (elements,))
    g.add("vals", "input", "f32", (elements,))
    g.add("off", "input", "i32", (rows + 1,))
    g.add("g", "gather", "f32", (elements,), args=("col", "x"))
    g.add("p", "map", "f32", (elements,), fn="mul2", args=("vals", "g"))
    g.add("y", "foldseg", "f32", (rows,), fn="add", args=("p", "off"), output=True)
    return g, fc.fc_plan(g, "bytes")


@pytest.mark.parametrize("elements", [4000000, (1 << 28) + 1, (1 << 29) - 1])          # what the fold that sorts its elements leaves to this one
def test_a_segmented_fold_takes_the_rows_it_took_without_the_operators_counters(elements):
    # four flags of 8 bytes for every 256 rows, in what the control block leaves behind its first 65792 bytes
    most = (B.FC_SCRATCH_CONTROL_BYTES - 256 - 65536) // 32 * 256
    for rows, blocked in ((66450000, True), (66500000, True), (most, True), (most + 1, False)):
        g, part = spmv_of_many_rows(rows, elements)
        assert ("column-blocked" in fc.fc_cluster_kernel(g, part, 0)) == blocked, rows
        assert (fc.fc_scratch_bytes(g, part) >= B.FC_SCRATCH_CONTROL_BYTES + 32 * rows) == blocked, rows
