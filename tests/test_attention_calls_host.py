"""Calls beside the sparse decode that are refused before any launch (no GPU needed)."""
import pytest
import torch

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


def test_a_workspace_that_is_not_one_piece_of_memory_is_not_used():
    """A view that repeats or skips bytes has as many elements as asked for, and less memory, or another one's between."""
    batch = T.RaggedBatch([900, 300], 8, 2, device="cpu")
    size = T.PromptAttention(batch, [20, 20]).workspace.numel()
    whole = torch.zeros(2 * size + 64, dtype=torch.uint8)
    assert T.PromptAttention(batch, [20, 20], workspace=whole).workspace is whole
    assert whole.data_ptr() % 16 == 0
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(size), whole[::2], whole[1:], whole[:size - 1], whole.float()):
        got = T.PromptAttention(batch, [20, 20], workspace=bad).workspace
        assert got is not bad and got.is_contiguous() and got.numel() == size and got.dtype is torch.uint8
