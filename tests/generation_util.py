"""Plain 64-bit implementations of the generation step's operators, for its tests: from the definitions in include/resq.h, in
numpy and torch on the CPU, sharing nothing with the library."""
import math

import numpy as np
import torch


def row_bytes(d, r):
    return r + (d - r) // 2 + 16


def decode_rows(rows, d, r):
    """float64 [..., d] values of uint8 [..., row bytes] compact rows."""
    rows = rows.cpu()
    low = r + (d - r) // 2
    par = rows[..., low:low + 16].clone(memory_format=torch.contiguous_format).view(torch.float32).double()
    out = torch.empty(*rows.shape[:-1], d, dtype=torch.float64)
    out[..., :r] = rows[..., :r].double() * par[..., 0:1] + par[..., 1:2]
    packed = rows[..., r:low].long()
    out[..., r::2] = (packed % 16).double() * par[..., 2:3] + par[..., 3:4]
    out[..., r + 1::2] = (packed // 16).double() * par[..., 2:3] + par[..., 3:4]
    return out


def plan(lens, news, free, taken, table, page, num_pages, cap):
    """(lens, cu_tokens, cu_pages, positions, slots, table, state) by loops; lists and a nested list for the table."""
    table = [list(t) for t in table]
    held = [-(-n // page) for n in lens]
    want = [-(-(n + a) // page) for n, a in zip(lens, news)]
    status = 0
    if taken < 0 or min(lens) < 0 or min(news) < 0:
        status = 4
    elif sum(news) > cap:
        status = 3
    elif max(want) > len(table[0]):
        status = 2
    elif taken + sum(w - h for w, h in zip(want, held)) > len(free):
        status = 1
    if status:
        zero = [0] * (len(lens) + 1)
        return list(lens), zero, zero, [0] * cap, [-1] * cap, table, [taken, status]
    cu, cp, positions, slots = [0], [0], [], []
    for b, (n, a) in enumerate(zip(lens, news)):
        for i in range(held[b], want[b]):
            table[b][i] = free[taken]
            taken += 1
        for t in range(n, n + a):
            p = table[b][t // page]
            positions.append(t)
            slots.append(p * page + t % page if 0 <= p < num_pages else -1)
        cu.append(cu[-1] + a)
        cp.append(cp[-1] + want[b] - held[b])
    pad = cap - len(slots)
    return [n + a for n, a in zip(lens, news)], cu, cp, positions + [0] * pad, slots + [-1] * pad, table, [taken, 0]


def rope(x, positions, freq, heads_q, w_q, w_k, eps, interleaved, mscale):
    """(float64 result, sum of the magnitudes that go into each element) of x [tokens, heads, d]."""
    n = x.cpu().double()
    if w_q is not None or w_k is not None:
        n = n / torch.sqrt(n.square().mean(-1, keepdim=True) + eps)
        if heads_q:
            n[:, :heads_q] *= w_q.cpu().double()
        if heads_q < n.shape[1]:
            n[:, heads_q:] *= w_k.cpu().double()
    y, size = n.clone(), n.abs()
    half = 0 if freq is None else len(freq)
    for i in range(half):
        ca, cb = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        # whole turns taken off in extended precision: np.longdouble has 64 bits of mantissa, fp64 products would lose
        # what this is there to check
        turns = np.asarray(positions.cpu().numpy(), dtype=np.longdouble) * np.longdouble(float(freq[i])) / (2 * np.longdouble(np.pi))
        angle = torch.from_numpy(((turns - np.rint(turns)) * 2 * np.longdouble(np.pi)).astype(np.float64))[:, None]
        a, b = n[..., ca], n[..., cb]
        y[..., ca], y[..., cb] = mscale * (a * angle.cos() - b * angle.sin()), mscale * (b * angle.cos() + a * angle.sin())
        size[..., ca] = size[..., cb] = abs(mscale) * (a.abs() + b.abs())
    return y, size


def attend(q, k_pages, v_pages, lens, table, r, scale, softcap=0.0, window=0):
    """float64 (out [B, H, d], lse [B, H], bound of |kernel's out - out| besides the rounding to bf16, bound of lse's).

    The bounds.  A score is a sum of d products of a bf16 query and a code (times a scale, plus the zero-point's term), exact
    products, sums in fp32 of terms that may carry an offset of 16 per code: at most 64 roundings of 2^-24 of the sum of the
    terms' magnitudes, 2^-18 of it, whatever their order.  tanh moves it by 2^-22 of the cap.  A weight e^(x - lse) is then off by twice that, and by 2^-15 of
    itself: 2^-16 for its two bf16 parts, the rest for the exponential and sums.  In the weighted sum codes may carry an offset of
    up to 143 quantization steps of the 4-bit group (255 of the 8-bit one)."""
    q, lens, table = q.cpu().double(), [int(n) for n in lens], table.cpu().long()
    pages, page, d = k_pages.shape[0], k_pages.shape[2], q.shape[-1]
    share = q.shape[1] // k_pages.shape[1]
    k_pages, v_pages = k_pages.cpu(), v_pages.cpu()
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    tol, tol_lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64)
    for b, n in enumerate(lens):
        n = min(max(n, 0), table.shape[1] * page)
        t = torch.arange(max(0, n - window) if window else 0, n)
        ids = table[b, t // page]
        t, ids = t[(ids >= 0) & (ids < pages)], ids[(ids >= 0) & (ids < pages)]
        if not len(t):
            continue
        for h in range(k_pages.shape[1]):
            kr, vr = k_pages[ids, h, t % page], v_pages[ids, h, t % page]
            k, v = decode_rows(kr, d, r), decode_rows(vr, d, r)
            low = r + (d - r) // 2
            steps = [x[..., low:low + 16].clone(memory_format=torch.contiguous_format).view(torch.float32).double() for x in (kr, vr)]
            up = lambda p, hi, lo: torch.cat((hi * p[:, 0:1].expand(-1, r), lo * p[:, 2:3].expand(-1, d - r)), 1).abs()
            kbig, vbig = k.abs() + up(steps[0], 256, 32), v.abs() + up(steps[1], 255, 143)
            for i in range(h * share, (h + 1) * share):
                x = scale * (k @ q[b, i])
                off = 2.0 ** -18 * scale * (kbig @ q[b, i].abs()).max()
                if softcap:
                    x = softcap * torch.tanh(x / softcap)
                    off = off + 2.0 ** -22 * softcap
                lse[b, i] = torch.logsumexp(x, 0)
                p = torch.exp(x - lse[b, i])
                out[b, i] = p @ v
                tol[b, i] = (2 * off + 2.0 ** -15) * (p @ vbig)
                tol_lse[b, i] = off + 2.0 ** -21 * (1 + lse[b, i].abs())
    return out, lse, tol, tol_lse


def make_pages(g, pages, heads, page, d, r, order="head", pad=0, device="cuda"):
    """uint8 [pages, heads, page, row bytes + pad] filled with plausible rows, in memory in that order, or with a token's heads
    together ("token")."""
    nb = row_bytes(d, r)
    rows = torch.randint(0, 256, (pages, heads, page, nb + pad), generator=g, dtype=torch.uint8)
    par = torch.empty(pages, heads, page, 4)
    par[..., 0] = 0.02 * torch.rand(pages, heads, page, generator=g) + 0.005
    par[..., 2] = 0.2 * torch.rand(pages, heads, page, generator=g) + 0.05
    par[..., 1] = -127 * par[..., 0] * (1 + 0.1 * torch.randn(pages, heads, page, generator=g))
    par[..., 3] = -7.5 * par[..., 2] * (1 + 0.1 * torch.randn(pages, heads, page, generator=g))
    rows[..., nb - 16:nb] = par.view(torch.uint8)
    rows = rows.to(device)
    return rows.transpose(1, 2).contiguous().transpose(1, 2) if order == "token" else rows
