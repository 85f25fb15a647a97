"""The step that the smoke run compares with the oracle: the comparison fails where an operator has not done its part."""
import numpy as np
import pytest

import __graft_entry__ as entry

OUTPUTS = ["table", "lengths_after", "row_start", "slots", "positions", "request", "cursor_after", "unplaced", "turned", "k_cache", "v_cache", "out"]


def test_the_oracle_s_own_step_passes_rounded_to_32_bits():
    s = entry.cache_step()
    want = entry.cache_step_by_oracle(s)
    assert set(OUTPUTS) | {"pool"} == set(want)
    assert all(a.dtype == (np.float32 if want[n].dtype == np.float64 else want[n].dtype) for n, a in s.items() if n in want)
    entry.check_cache_step({n: a.astype(s[n].dtype) for n, a in want.items()}, want)


@pytest.mark.parametrize("missing", OUTPUTS)
def test_an_output_left_as_it_was_fails(missing):
    s = entry.cache_step()
    want = entry.cache_step_by_oracle(s)
    with pytest.raises(AssertionError, match=missing):
        entry.check_cache_step({**want, missing: s[missing]}, want)


@pytest.mark.parametrize("missing", ["q_weight", "k_weight", "cos_sin"])
def test_heads_without_their_norm_or_their_rotation_fail(missing):
    s = entry.cache_step()
    want = entry.cache_step_by_oracle(s)
    plain = np.ones_like(s[missing])
    if missing == "cos_sin":
        plain[:, plain.shape[1] // 2:] = 0
    with pytest.raises(AssertionError, match="turned|k_cache"):
        entry.check_cache_step(entry.cache_step_by_oracle({**s, missing: plain}), want)


def test_a_step_that_stored_nothing_fails_though_its_attention_fits_what_is_there():
    s = entry.cache_step()
    want = entry.cache_step_by_oracle(s)
    nothing = {**want, "table": s["table"], "k_cache": s["k_cache"], "v_cache": s["v_cache"], "out": np.zeros_like(want["out"])}
    with pytest.raises(AssertionError):
        entry.check_cache_step(nothing, want)
