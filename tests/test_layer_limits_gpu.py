"""The operators around a layer's products on the GPU where their arguments come to an end: arrays that no plan gives, numbers far from the usual."""
import math

import pytest
import torch

import layer_util as plain
from test_layer_gpu import DEV, gen, heads, ints, rq, sums   # noqa: F401

pytestmark = pytest.mark.gpu


def guarded(shape, dtype, room=4096):
    """A tensor in the middle of a larger one, and what says whether that is as it was around it."""
    n = math.prod(shape)
    whole = torch.full((n + 2 * room,), 7.0, dtype=dtype, device=DEV)
    return whole[room:room + n].view(shape), lambda: bool((whole[:room] == 7).all()) and bool((whole[room + n:] == 7).all())


@pytest.mark.parametrize("cu_q,cu_k", [([30, 10, 40, 5], [0, 50, 20, 60]), ([40, 0, 40, 0], [50, 0, 50, 0]), ([5, 3, 2, -9], [9, 4, 70, 2])])
def test_prompts_lengths_that_decrease(rq, cu_q, cu_k):   # noqa: F811
    g = gen(2)
    for d in (64, 128):
        q, k, v = heads(g, 40, 2, d), heads(g, 50, 2, d), heads(g, 50, 2, d)
        (out, out_kept), (lse, lse_kept) = guarded((40, 2, d), torch.bfloat16), guarded((40, 2), torch.float32)
        rq.resq_attend_prompts(q, k, v, ints(cu_q), ints(cu_k), out=out, lse=lse)
        torch.cuda.synchronize()
        assert out_kept() and lse_kept()


def test_prompts_lengths_that_decrease_beyond_32_bits(rq):   # noqa: F811
    """65535 sequences of up to 4 million queries: more rows than 32 bits count in all."""
    tokens, share, batch = 1 << 22, 8, 65535
    q = torch.zeros(tokens, share, 8, dtype=torch.bfloat16, device=DEV)
    k = heads(gen(3), 64, 1, 8)
    (out, out_kept), (lse, lse_kept) = guarded((tokens, share, 8), torch.bfloat16), guarded((tokens, share), torch.float32)
    cu_q = ints([0, tokens]).repeat(batch // 2 + 1)
    for cu_k in (ints([0, 64]).repeat(batch // 2 + 1), ints([64, 0]).repeat(batch // 2 + 1)):
        rq.resq_attend_prompts(q, k, k, cu_q, cu_k, out=out, lse=lse)
        torch.cuda.synchronize()
        assert out_kept() and lse_kept()
