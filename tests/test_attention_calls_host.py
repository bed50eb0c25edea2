"""Calls beside the sparse decode that are refused before any launch (no GPU needed)."""
import pytest

import paper_2502_12216_amd as T
from paper_2502_12216_amd import _capi as C
from tests.test_attention_host import prompt, scored, shared, weights


@pytest.mark.parametrize("call", [prompt, weights, scored, shared])
@pytest.mark.parametrize("cap", [2.0 ** -121, 1e-40, 2.0 ** 121, 3e38])
def test_caps_that_leave_the_normal_numbers(call, cap):
    assert call(mod=C.ScoreMod(cap)) == 1
    assert b"cap" in C.lib().tactic_last_error()
    with pytest.raises(ValueError, match="cap"):
        T.ScoreMod(cap=cap)


@pytest.mark.parametrize("cap", [0.0, 2.0 ** -120, 1e-6, 50.0, 2.0 ** 120])
def test_caps_at_the_ends_of_their_range(cap):
    T.ScoreMod(cap=cap)
    assert scored(mod=C.ScoreMod(cap), n=1000) == 3  # the next check: the workspace
