"""Calls of the operators around a layer's products at the ends of what they take, without a GPU."""
import random

import pytest

from paper_2412_14363_amd import binding
from test_layer_cpu import BUFFER, PROMPTS, SHAPE, call


@pytest.mark.parametrize("change", [dict(ldk=1 << 24), dict(ldv=1 << 30), dict(ldk=(1 << 40) + 4, ldv=1 << 41), dict(heads_q=2, heads_k=1, ldkh=1 << 40, ldvh=3)])
def test_prompts_strides_that_are_never_taken(change):
    """One key's distance to the next, and one head's, mean nothing (torch gives any number there); a call with too small a workspace
    shows that nothing else is refused."""
    assert call("resq_attend_prompts", PROMPTS, tokens_k=1, nbytes=8, **change) == BUFFER


def test_prompts_strides_that_are_taken():
    for change in (dict(ldk=1 << 24), dict(ldv=1 << 24)):
        assert call("resq_attend_prompts", PROMPTS, tokens_k=2, nbytes=8, **change) == SHAPE


def test_prompts_of_any_number_that_is_allowed():
    """tokens_q * heads_q + 255 B heads_k < 2^31, as far as a launch counts its threads: taken below it, whatever the shares are, and refused not far above."""
    f = binding.resq_attend_prompts_workspace_bytes
    rng = random.Random(1)
    for _ in range(3000):
        batch, heads_k, share, d = (rng.choice([1, 2, 100, 65535]), rng.choice([1, 8, 33, 200, 4000]), rng.choice([1, 4, 7]), rng.choice([8, 64, 72, 128, 256]))
        left = (1 << 31) - 1 - 255 * batch * heads_k
        tokens = min(left // (heads_k * share), (1 << 30), ((1 << 31) - 65537) // (heads_k * share))
        if tokens >= 0 and heads_k * share <= 65535:
            assert f(tokens, 1000, batch, heads_k * share, heads_k, d) > 0, (tokens, batch, heads_k, share, d)
    assert f(1, 1, 65535, 200, 200, 128) == f(1, 1, 65535, 400, 400, 64) == 0
