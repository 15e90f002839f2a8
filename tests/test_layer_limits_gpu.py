"""The operators around a layer's products on the GPU where their arguments come to an end: arrays that no plan gives, numbers far from the usual."""
import math

import pytest
import torch

import layer_util as plain
from test_layer_gpu import DEV, gen, heads, ints, prefix_inputs, rq   # noqa: F401

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


# ---- capped scores ------------------------------------------------------------------------------------
# Off by 2^-19.9 of themselves at most: two polynomials of four steps with terms of one sign, a rounding of 2^-24 for each (8), one of the
# numerator's constants, the reciprocal's last place (2) and the quotient's rounding (1), the argument's square, nine roundings of which at most
# half reach the quotient (4.5), and the fit (0.3): 16.8 roundings.  A weight is off by twice that.

def capped(want, exact, most):
    """(results with the cap, bounds): those without it, in whose place the cap puts its own error and no other; scores below `most`."""
    out, lse, tol, tol_lse = want
    off = 2.0 ** -19.9 * most
    return out, lse, tol + 2 * off * exact, tol_lse + off


@pytest.mark.parametrize("cap", [1e4, 1e6, 1e8, 1.5e38, 3.4e38])
@pytest.mark.parametrize("d,window", [(64, 0), (128, 50), (200, 0)])
def test_prompts_caps_far_above_the_scores(rq, d, window, cap):   # noqa: F811
    g, cu_q, cu_k = gen(d), [0, 70, 75, 200], [0, 90, 95, 320]
    q, k, v = heads(g, 200, 4, d), heads(g, 320, 2, d), heads(g, 320, 2, d)
    out, lse = torch.empty_like(q), torch.empty(200, 4, device=DEV)
    rq.resq_attend_prompts(q, k, v, ints(cu_q), ints(cu_k), softcap=cap, window=window, out=out, lse=lse)
    without = plain.prompts(q, k, v, cu_q, cu_k, d ** -0.5, 0.0, window)   # its bounds know nothing of a cap
    want = plain.prompts(q, k, v, cu_q, cu_k, d ** -0.5, cap, window)
    most = 20.0
    assert float((q.float().norm(dim=2).max() * k.float().norm(dim=2).max()) * d ** -0.5) < 2 * most
    plain.check(out, lse, capped((want[0], want[1], without[2] * 1.01, without[3] * 1.01), v.double().abs().amax().cpu(), 2 * most))


@pytest.mark.parametrize("cap", [1e4, 1e6, 1e8, 1.5e38, 3.4e38])
@pytest.mark.parametrize("d,r,window", [(64, 8, 0), (128, 16, 150), (256, 32, 0)])
def test_prefix_caps_far_above_the_scores(rq, d, r, window, cap):   # noqa: F811
    i = prefix_inputs(300, [0, 1, 40, -1], 4, 2, d, r, 16, seed=d)
    args = i["q"], i["k_pages"], i["v_pages"], 300, i["prefix_table"], i["lens"], i["block_table"], r, d ** -0.5
    without, want = plain.prefix(*args, 0.0, window), plain.prefix(*args, cap, window)
    lse = torch.empty(4, 4, device=DEV)
    out = rq.resq_attend_kv_prefix(**i, softcap=cap, window=window, lse=lse)
    live = want[1][torch.isfinite(want[1])]
    most = float(live.abs().max()) + 8   # a log of a few hundred exponentials is no more than that below the largest score
    plain.check(out, lse, capped((want[0], want[1], without[2] * 1.01, without[3] * 1.01), want[0].abs().max() + 8, most))


@pytest.mark.parametrize("cap", [1e-30, 0.5, 5.0, 50.0, 1e3, 1e5])
@pytest.mark.parametrize("d", [64, 128])
def test_log_sum_exps_of_one_capped_score(rq, d, cap):   # noqa: F811
    """A query that sees one key has its score as log-sum-exp: small scores, scores about the cap, far above it, and of either sign."""
    g, n = gen(7), 400
    q, k = heads(g, n, 2, d), heads(g, n, 2, d)
    k *= torch.exp(torch.linspace(-12, 12, n, device=DEV))[:, None, None].to(torch.bfloat16)
    lse = torch.empty(n, 2, device=DEV)
    rq.resq_attend_prompts(q, k, k, ints([0, n]), softcap=cap, window=1, lse=lse)
    x, size = ((a * b).sum(-1) * d ** -0.5 for a, b in ((q.cpu().double(), k.cpu().double()), (q.cpu().double().abs(), k.cpu().double().abs())))
    want = cap * torch.tanh(x / cap)
    # what the score itself may be off by, as far as the cap lets it through; the cap's error and three roundings of constants.  Then m ln 2 + ln w of
    # w = 2^(x - m), where m may be up to 8 below x: that difference (2^-22), the exponential (2^-23), a logarithm below 5.6 (2^-21) and two
    # roundings of m ln 2, 5.6 of which x does not account for (2^-20.5): 2^-19.3
    off = d * 2.0 ** -24 * size + 2.0 ** -22 * x.abs()
    through = torch.maximum(cap * torch.tanh((x + off) / cap) - want, want - cap * torch.tanh((x - off) / cap))
    tol = through + (2.0 ** -19.9 + 2.0 ** -22) * want.abs() + 2.0 ** -19.3
    over = (lse.cpu().double() - want).abs() - tol
    assert bool((over <= 0).all()), (float(over.max()), float(cap))


def test_caps_of_scores_that_are_not_numbers(rq):   # noqa: F811
    """A NaN among the keys that a row sees is one in its result, capped or not, and nothing to the others."""
    g, n = gen(5), 200
    q, k, v = (heads(g, n, 1, 64) for _ in range(3))
    k[100, 0, 3] = math.nan
    for cap in (0.0, 1.0, 30.0, 1e4):
        lse = torch.empty(n, 1, device=DEV)
        out = rq.resq_attend_prompts(q, k, v, ints([0, n]), softcap=cap, lse=lse)
        assert bool(torch.isfinite(out[:100]).all()) and bool(torch.isfinite(lse[:100]).all())
        assert bool(torch.isnan(out[100:]).all()) and bool(torch.isnan(lse[100:]).all())


# ---- values that are not finite and weigh next to nothing -------------------------------------------------

@pytest.mark.parametrize("hk", [1, 300])   # keys in parts, and in one
def test_prompts_values_that_are_seen_and_weigh_nothing(rq, hk):   # noqa: F811
    """NaN times a weight is NaN however small the weight is, and however the keys are cut."""
    g, n = gen(1), 1500
    q = torch.ones(2, hk, 8, dtype=torch.bfloat16, device=DEV)
    k, v = torch.full((n, hk, 8), -30.0, dtype=torch.bfloat16, device=DEV), heads(g, n, hk, 8)
    k[1000:] = 30   # e^-480 of these is what the first ones weigh
    v[10, :, 3], v[1200, :, 5] = math.nan, math.nan
    for window in (0, 600):
        out = rq.resq_attend_prompts(q, k, v, ints([0, 2]), ints([0, n]), scale=1.0, window=window)
        bad = torch.isnan(out)
        assert bool(bad[..., 5].all()) and bool((bad[..., 3] == (window == 0)).all()) and not bool(bad[..., [0, 1, 2, 4, 6, 7]].any())


@pytest.mark.parametrize("n,batch,hk", [(500, 3, 1), (500, 3, 300), (100, 3, 1)])   # the prefix in parts, in one
def test_prefix_values_that_are_seen_and_weigh_nothing(rq, n, batch, hk):   # noqa: F811
    i = prefix_inputs(n, [0, 5, 60], hk, hk, 16, 8, 16)
    low, t = 8 + 4, i["prefix_table"].cpu()
    i["q"].fill_(1)
    for tok in range(n):
        par = i["k_pages"][int(t[tok // 16]), :, tok % 16, low:low + 16]
        z = -20.0 if tok < n // 2 else 20.0
        par.copy_(torch.tensor([0.0, z, 0.0, z]).view(torch.uint8).to(DEV))
    spot = i["v_pages"][int(t[10 // 16]), :, 10 % 16]
    spot[:, low:low + 4] = torch.tensor([math.nan]).view(torch.uint8).to(DEV)   # the 8-bit group's scale
    for window in (0, n // 2):
        out = rq.resq_attend_kv_prefix(**i, scale=1.0, window=window)
        bad = torch.isnan(out)
        assert bool((bad[..., :8] == (window == 0)).all()) and not bool(bad[..., 8:].any())


# ---- norms of numbers far from 1 -------------------------------------------------------------------------

@pytest.mark.parametrize("size", [1e-18, 1e-19, 3e-20, 1e-21, 1e-22])
@pytest.mark.parametrize("width", [64, 4096])
def test_norm_of_small_rows_without_eps(rq, width, size):   # noqa: F811
    """Mean squares below the smallest normal number of fp32, 1.2e-38, hold 2^-149 steps: of 1e-44 some two digits are left."""
    i = dict(y=None, h=(torch.rand(3, width, generator=gen(width)) + 0.5).to(DEV) * size, w_pre=torch.ones(width, dtype=torch.bfloat16, device=DEV))
    x = rq.resq_norm_residual(**i, eps=0.0)[1]
    want = plain.norm_residual(**i, w_post=None, gate=None, alpha=1.0, eps=0.0, offset=0.0)[1]
    step = 2.0 ** -149 / (size * size)   # of a mean square; a sum's terms are rounded to it, each by half a step of the 1.08 they are
    off = 2.0 ** -17 + min(64 * step, 1.0)
    over = (x.cpu().double() - want).abs() - want * (off + 2.0 ** -8)
    assert bool((over <= 0).all()), float(over.max())
