"""Calls of the operators around a layer's products at the ends of what they take, without a GPU."""
import pytest

from test_layer_cpu import BUFFER, PROMPTS, SHAPE, call


@pytest.mark.parametrize("change", [dict(ldk=1 << 24), dict(ldv=1 << 30), dict(ldk=(1 << 40) + 4, ldv=1 << 41), dict(heads_q=2, heads_k=1, ldkh=1 << 40, ldvh=3)])
def test_prompts_strides_that_are_never_taken(change):
    """One key's distance to the next, and one head's, mean nothing (torch gives any number there); a call with too small a workspace
    shows that nothing else is refused."""
    assert call("resq_attend_prompts", PROMPTS, tokens_k=1, nbytes=8, **change) == BUFFER


def test_prompts_strides_that_are_taken():
    for change in (dict(ldk=1 << 24), dict(ldv=1 << 24)):
        assert call("resq_attend_prompts", PROMPTS, tokens_k=2, nbytes=8, **change) == SHAPE
