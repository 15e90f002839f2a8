"""Plain 64-bit implementations of the operators around a layer's products, for their tests: from the definitions in include/resq.h, in torch
on the CPU, sharing nothing with the library."""
import math

import torch


def rows(q, k, v, first, last, scale, cap, weight_step):
    """One head: queries [n, d] over keys first[i] <= j < last[i] -> (out [n, d], lse [n], bound of the kernel's error before its last
    rounding, bound of lse's), all in 64 bits.

    The bounds.  A score is a sum of d products, each exact in fp32, of at most d roundings of 2^-24 of its terms' magnitudes; its
    product with the scale, its difference from the maximum and the exponential's argument are three more, of the score and the
    maximum; cap tanh(x / cap) as cap (1 - 2 / (1 + e^(2 x / cap))) is off by 2^-21 of the cap: 2^-22 for the reciprocal's last place, 2^-23 for
    the sum's and the exponential's, which the slope of 1 / (1 + e), at most 1 / 4 of e's relative error, makes smaller, 2^-23 for the rest.  A weight is off by twice what its score is (its own and the sum's), by its rounding
    as an operand (weight_step, half a step of that type) and by 2^-21 for the exponential and the quotient.  The weighted sum has at
    most as many roundings of 2^-24 as there are keys."""
    x = scale * (q @ k.T)
    size = scale * (q.abs() @ k.abs().T)
    t = torch.arange(len(k))
    seen = (t >= first[:, None]) & (t < last[:, None])
    some = seen.any(1)
    off = torch.where(seen, q.shape[1] * 2.0 ** -24 * size + 2.0 ** -22 * x.abs(), 0.0)
    if cap:
        x = cap * torch.tanh(x / cap)
        off = off + 2.0 ** -21 * cap
    x = torch.where(seen, x, -math.inf)
    off = (off.nan_to_num().amax(1) if len(k) else torch.zeros(len(q), dtype=torch.float64)) + 2.0 ** -22 * torch.where(
        some, x.amax(1) if len(k) else 0.0, 0.0).abs()
    lse = torch.logsumexp(x, 1) if len(k) else torch.full((len(q),), -math.inf, dtype=torch.float64)
    p = torch.where(some[:, None], torch.exp(x - lse[:, None]), 0.0)
    v = torch.where(seen.any(0)[:, None], v, 0.0)
    out, mag = p @ v, p @ v.abs()
    step = 2 * off + weight_step + 2.0 ** -21 + 2.0 ** -24 * len(k)
    return out, lse, step[:, None] * mag, off + 2.0 ** -21 * (1 + lse.abs()) + 2.0 ** -24 * len(k)


def prompts(q, k, v, cu_q, cu_k, scale, cap=0.0, window=0):
    """resq_attend_prompts: (out, lse, bounds of both) like rows(); NaN for rows outside of the sequences."""
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    share = q.shape[1] // k.shape[1]
    out, tol = torch.full_like(q, math.nan), torch.full_like(q, math.nan)
    lse, tol_lse = torch.full(q.shape[:2], math.nan, dtype=torch.float64), torch.full(q.shape[:2], math.nan, dtype=torch.float64)
    for q0, q1, k0, k1 in zip(cu_q, cu_q[1:], cu_k, cu_k[1:]):
        last = torch.arange(q1 - q0) + (k1 - k0) - (q1 - q0) + 1
        first = last - window if window else 0 * last
        for h in range(q.shape[1] if q1 > q0 else 0):
            got = rows(q[q0:q1, h], k[k0:k1, h // share], v[k0:k1, h // share], first, last, scale, cap, 2.0 ** -8)
            out[q0:q1, h], lse[q0:q1, h], tol[q0:q1, h], tol_lse[q0:q1, h] = got
    return out, lse, tol, tol_lse


def check(got, got_lse, want, where=None):
    """bf16 results and fp32 sums against rows()' bounds; `where`: the rows to look at (all where None)."""
    out, lse, tol, tol_lse = want
    got, got_lse = got.detach().cpu().double(), None if got_lse is None else got_lse.cpu().double()
    if where is not None:
        got, out, tol, lse, tol_lse = got[where], out[where], tol[where], lse[where], tol_lse[where]
        got_lse = None if got_lse is None else got_lse[where]
    over = (got - out).abs() - (tol + 2.0 ** -8 * (out.abs() + tol) + 2.0 ** -133)
    assert bool((over <= 0).all()), (float(over.max()), torch.nonzero(~(over <= 0))[:5].tolist())
    if got_lse is not None:
        empty = lse == -math.inf
        assert bool((got_lse[empty] == -math.inf).all())
        over = ((got_lse - lse).abs() - tol_lse)[~empty]
        assert bool((over <= 0).all()), float(over.max())


def norm_residual(y, h, w_pre, w_post, gate, alpha, eps, offset):
    """resq_norm_residual: (h', x, bounds of the kernel's errors before its last roundings), in 64 bits.

    The bounds.  A mean square is a sum of squares, all of one sign: each term is rounded at most 64 times (32 in a thread, the rest
    between them, the quotient), its root halves that, and the root itself is off by 2^-23: 2^-18 + 2^-23 of the value, below 2^-17.
    The products behind it are a few roundings of 2^-24 more."""
    h = h.detach().cpu().double()
    out, off = h, torch.zeros_like(h)
    if y is not None:
        a = y.detach().cpu().double()
        if w_post is not None:
            a = a / torch.sqrt((a * a).mean(1, keepdim=True) + eps) * (offset + w_post.cpu().double())
        if gate is not None:
            a = a * gate.cpu().double()
        out = h + alpha * a
        off = 2.0 ** -17 * (alpha * a).abs() + 2.0 ** -23 * (h.abs() + (alpha * a).abs())
    if w_pre is None:
        return out, None, off, None
    f = (offset + w_pre.cpu().double()) / torch.sqrt((out * out).mean(1, keepdim=True) + eps)
    # what h' is off by moves the root by no more than it moves the largest row norm
    root = (off.square().mean(1, keepdim=True) / ((out * out).mean(1, keepdim=True) + eps)).sqrt()
    return out, out * f, off, (out * f).abs() * (root + 2.0 ** -17 + 2.0 ** -22) + off * f.abs()


def check_norm(h, x, want, wide):
    out, y, off, off_x = want
    if h is not None:
        over = (h.cpu().double() - out).abs() - (off + (2.0 ** -24 if wide else 2.0 ** -8) * (out.abs() + off) + 2.0 ** -133)
        assert bool((over <= 0).all()), float(over.max())
    if x is not None:
        over = (x.cpu().double() - y).abs() - (off_x + 2.0 ** -8 * (y.abs() + off_x) + 2.0 ** -133)
        assert bool((over <= 0).all()), float(over.max())


def prefix(q, k_pages, v_pages, prefix_len, prefix_table, lens, table, r, scale, cap=0.0, window=0):
    """resq_attend_kv_prefix: (out, lse, bounds of both).  The prefix's values are off by 2^-11 of themselves (half a step of fp16), its
    keys, two such numbers each, by 2^-22, both by 2^-38 of the largest one; the own tokens' code products may carry offsets of up to 143 steps, 255 of the 8-bit group, and
    their weights are two bf16 numbers: both are below what this takes for all tokens."""
    from generation_util import decode_rows
    q = q.cpu().double()
    d, page, pages = q.shape[-1], k_pages.shape[2], k_pages.shape[0]
    share = q.shape[1] // k_pages.shape[1]
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64)
    n = min(max(int(prefix_len), 0), len(prefix_table) * page)

    def there(ids, count):
        t = torch.arange(count)
        ids = ids.cpu().long()[t // page]
        ok = (ids >= 0) & (ids < pages)
        return ids[ok] * page + (t % page)[ok], t[ok]
    front, front_t = there(prefix_table, n)
    flat = [p.cpu().permute(0, 2, 1, 3).reshape(pages * page, *p.shape[1:2], p.shape[3]) for p in (k_pages, v_pages)]
    for b, own in enumerate(int(x) for x in lens):
        if own < 0:
            continue
        own = min(own, table.shape[1] * page)
        back, back_t = there(table[b], own)
        at, t = torch.cat((front, back)), torch.cat((front_t, back_t + n))
        if window:
            at = at[t >= n + own - window]
        if not len(at):
            continue
        for h in range(k_pages.shape[1]):
            rows_k, rows_v = (f[at, h] for f in flat)
            k, v = decode_rows(rows_k, d, r), decode_rows(rows_v, d, r)
            low = r + (d - r) // 2
            big = []
            for x, rows_x in ((k, rows_k), (v, rows_v)):
                s = rows_x[:, low:low + 16].clone(memory_format=torch.contiguous_format).view(torch.float32).double().abs()
                big.append(x.abs() + torch.cat((255 * s[:, 0:1].expand(-1, r), 143 * s[:, 2:3].expand(-1, d - r)), 1))
            for i in range(h * share, (h + 1) * share):
                x = scale * (k @ q[b, i])
                size = scale * ((k.abs() @ q[b, i].abs()) * 2.0 ** -22 + (big[0] @ q[b, i].abs()) * 2.0 ** -18 +
                                2.0 ** -38 * k.abs().max() * q[b, i].abs().sum())
                off = (size + 2.0 ** -22 * x.abs()).max() + 2.0 ** -22 * x.max().abs()
                if cap:
                    x = cap * torch.tanh(x / cap)
                    off = off + 2.0 ** -21 * cap
                lse[b, i] = torch.logsumexp(x, 0)
                p = torch.exp(x - lse[b, i])
                out[b, i] = p @ v
                step = 2 * off + 2.0 ** -15 + 2.0 ** -24 * len(at)
                tol[b, i] = step * (p @ big[1]) + 2.0 ** -10 * (p @ v.abs()) + 2.0 ** -35 * v.abs().sum(0) + 2.0 ** -38 * v.abs().max()
                tol_lse[b, i] = off + 2.0 ** -21 * (1 + lse[b, i].abs()) + 2.0 ** -24 * len(at)
    return out, lse, tol, tol_lse
