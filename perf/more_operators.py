"""The operators that stand around a layer's products when a model reads prompts and when many answers grow from one prompt: attention
over whole prompts (causal, packed sequences, grouped heads, behind cached tokens or not), attention of one new token per sequence
over a prefix that all sequences of the batch share and their own tokens behind it (both in the paged compact K/V cache), and the
norms before and after a block with its gate, its residual scale and the residual sum.

``run`` computes them from elementary torch operations in 32 bits where ``own`` is false, and calls
``paper_2412_14363_amd.binding`` where it is true.
"""
import math
import random

import torch

own = False
DEV = "cuda"


# ---- the cases ---------------------------------------------------------------------------------

def listed():
    return [
        # the smallest prompt: a question of 17 tokens on an 8B model's heads, queries, keys and values as the projection wrote them
        {"name": "prompt_b1_17", "op": "prompt", "batch": 1, "longest": 17, "old": 0, "hq": 32, "hk": 8, "d": 128, "window": 0, "cap": 0.0,
         "pad": 0},
        # an ordinary prompt of the same model
        {"name": "prompt_b1_2048", "op": "prompt", "batch": 1, "longest": 2048, "old": 0, "hq": 32, "hk": 8, "d": 128, "window": 0, "cap": 0.0,
         "pad": 0},
        # one long document
        {"name": "prompt_b1_8192", "op": "prompt", "batch": 1, "longest": 8192, "old": 0, "hq": 32, "hk": 8, "d": 128, "window": 0, "cap": 0.0,
         "pad": 0},
        # a packed batch of ragged prompts, padded behind the last: heads of 64 without sharing, a window, capped scores
        {"name": "prompt_b24_window_cap", "op": "prompt", "batch": 24, "longest": 3001, "old": 0, "hq": 12, "hk": 12, "d": 64, "window": 1500,
         "cap": 30.0, "pad": 77},
        # the next chunks of three long documents behind what the cache has of them, on a 70B model's heads
        {"name": "prompt_b3_behind_30000", "op": "prompt", "batch": 3, "longest": 300, "old": 30000, "hq": 64, "hk": 8, "d": 128, "window": 0,
         "cap": 0.0, "pad": 0},
        # four answers to one question: the smallest batch that shares anything worth it
        {"name": "prefix_b4_1000", "op": "prefix", "batch": 4, "prefix": 1000, "longest": 60, "hq": 32, "hk": 8, "d": 128, "r": 16, "page": 16,
         "order": "head", "window": 0, "cap": 0.0},
        # 64 requests behind the same instructions, answers and questions of ragged lengths
        {"name": "prefix_b64_8192", "op": "prefix", "batch": 64, "prefix": 8192, "longest": 900, "hq": 32, "hk": 8, "d": 128, "r": 16, "page": 16,
         "order": "head", "window": 0, "cap": 0.0},
        # 200 requests about one long document, a prefix that ends inside a page, on a 70B model's heads
        {"name": "prefix_b200_30001", "op": "prefix", "batch": 200, "prefix": 30001, "longest": 300, "hq": 64, "hk": 8, "d": 128, "r": 16,
         "page": 64, "order": "head", "window": 0, "cap": 0.0},
        # heads of 64 without sharing, odd pages that keep a token's heads together, a window that ends inside the prefix, capped scores
        {"name": "prefix_b33_window_cap", "op": "prefix", "batch": 33, "prefix": 5000, "longest": 400, "hq": 12, "hk": 12, "d": 64, "r": 8,
         "page": 24, "order": "token", "window": 3500, "cap": 30.0},
        # one new token between two blocks of an 8B model: residual sum and the next block's norm
        {"name": "norm_m1_4096", "op": "norm", "tokens": 1, "width": 4096, "post": False, "gate": "none", "wide": False, "alpha": 1.0,
         "offset": 0.0},
        # a ragged prefill batch of a 70B model, with a norm behind the block too, weights stored as their distance from one
        {"name": "norm_m3001_8192_post", "op": "norm", "tokens": 3001, "width": 8192, "post": True, "gate": "none", "wide": False, "alpha": 1.0,
         "offset": 1.0},
        # the same width with the residual stream in 32 bits, a gate for each token and a residual scale
        {"name": "norm_m8192_8192_gate", "op": "norm", "tokens": 8192, "width": 8192, "post": True, "gate": "token", "wide": True, "alpha": 0.22,
         "offset": 0.0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["prompt", "prompt", "prefix", "prefix", "norm"])
    d = rng.choice([64, 128, 128, 128, 256, 96, 8 * rng.randint(2, 32)])
    hk = rng.choice([1, 2, 4, 8, 8, 12])
    share = rng.choice([1, 1, 2, 4, 4, 7, 8])
    cap = rng.choice([0.0, 0.0, 20.0, 50.0])
    if op == "prompt":
        batch = rng.choice([1, 1, _log_int(rng, 1, 48)])
        pairs = 8192 * 8192 * 32 * 128 // (batch * hk * share * max(d, 128)) // 2   # of queries and keys of a sequence, at most
        longest = _log_int(rng, 1, min(16000, math.isqrt(pairs)))
        old = rng.choice([0, 0, _log_int(rng, 1, max(1, min(40000, pairs // longest - longest)))])
        return {"op": op, "batch": batch, "longest": longest, "old": old, "hq": hk * share, "hk": hk, "d": d,
                "window": rng.choice([0, 0, 0, _log_int(rng, 1, 8192)]), "cap": cap, "pad": rng.choice([0, 0, rng.randint(1, 200)])}
    if op == "prefix":
        batch = _log_int(rng, 1, 256)
        most = 200 * 64 * 30000 * 128 // (batch * hk * share * max(d, 128))
        prefix = _log_int(rng, 1, max(2, min(60000, most // 2)))
        longest = rng.choice([1, _log_int(rng, 1, max(2, min(1000, most // 4)))])
        r = rng.choice([d // 8 // 8 * 8, 0, d, rng.randrange(0, d + 1, 8), rng.randrange(0, d + 1, 8)])
        return {"op": op, "batch": batch, "prefix": prefix, "longest": longest, "hq": hk * share, "hk": hk, "d": d, "r": r,
                "page": rng.choice([16, 16, 32, 64, 128, 8, 24, rng.randint(1, 100)]), "order": rng.choice(["head", "head", "token"]),
                "window": rng.choice([0, 0, 0, _log_int(rng, 1, 8192)]), "cap": cap}
    width = rng.choice([4096, 8192, 5120, _log_int(rng, 64, 16384), 8 * _log_int(rng, 8, 2048)])
    return {"op": op, "tokens": _log_int(rng, 1, 8192 * 8192 // max(width, 1024)), "width": width, "post": rng.random() < 0.5,
            "gate": rng.choice(["none", "none", "channel", "token"]), "wide": rng.random() < 0.4, "alpha": rng.choice([1.0, 1.0, 0.22, 1.5]),
            "offset": rng.choice([0.0, 0.0, 1.0])}


# ---- what a case's lengths are (its work goes by them; the seed makes everything else) -----------------------------

def _news(c):
    """New tokens of each prompt: `longest` for one, ragged below it for the others."""
    rng = random.Random(c["batch"] * 1000003 + c["longest"])
    more = [rng.choice([0] + [rng.randint(1, c["longest"])] * 15) for _ in range(c["batch"] - 1)]
    at = rng.randint(0, len(more))
    return more[:at] + [c["longest"]] + more[at:]


def _olds(c):
    """Tokens that the cache has of each prompt already."""
    rng = random.Random(c["batch"] * 1000033 + c["old"])
    return [c["old"]] + [rng.randint(0, c["old"]) for _ in range(c["batch"] - 1)]


def _lens(c):
    """Own tokens of each sequence behind the shared prefix, some without any yet."""
    rng = random.Random(c["batch"] * 1000037 + c["longest"])
    return [c["longest"]] + [rng.choice([0] + [rng.randint(1, c["longest"])] * 15) for _ in range(c["batch"] - 1)]


def _row_bytes(d, r):
    return r + (d - r) // 2 + 16


# ---- inputs ------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _sums(values):
    got = [0]
    for v in values:
        got.append(got[-1] + v)
    return got


def _pick(g, n, k):
    """k different whole numbers below n, in any order."""
    return torch.randperm(n, generator=g, device=DEV)[:k].to(torch.int32)


def _heads(g, *shape, r=0):
    """bf16 head vectors; the first r channels, the ones that are kept in 8 bits, vary most."""
    x = torch.randn(*shape, generator=g, device=DEV)
    x += 0.3 * torch.randn(shape[-1], generator=g, device=DEV)
    x[..., :r] *= 3.0
    return x.to(torch.bfloat16)


def _quantize(x, levels):
    """Codes, scale and zero-point of each row."""
    z = x.amin(-1, keepdim=True)
    span = x.amax(-1, keepdim=True) - z
    scale = torch.where(span == 0, 1.0, span / levels)
    return ((x - z) / scale).round().clamp(0, levels), scale, z


def _pages(g, n, heads, page, d, r, order):
    """Cache pages [n, heads, page, row bytes] of quantized heads, in memory in that order or with a token's heads together: 8-bit
    codes, pairs of 4-bit codes, then both groups' scale and zero-point."""
    x = _heads(g, n, heads, page, d, r=r).float()
    one = torch.ones(n, heads, page, 1, device=DEV)
    got, par = [], []
    if r:
        q, *p = _quantize(x[..., :r], 255)
        got, par = [q.to(torch.uint8)], p
    else:
        par = [one, 0 * one]
    if r < d:
        q, *p = _quantize(x[..., r:], 15)
        q = q.to(torch.uint8)
        got.append(q[..., 0::2] | (q[..., 1::2] << 4))
        par = par + p
    else:
        par = par + [one, 0 * one]
    rows = torch.cat(got + [torch.cat(par, -1).contiguous().view(torch.uint8)], -1)
    return rows.transpose(1, 2).contiguous().transpose(1, 2) if order == "token" else rows


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = {"c": c, "kept": {}}
    if c["op"] == "prompt":
        news, olds = _news(c), _olds(c)
        cu_q, cu_k = _sums(news), _sums([n + o for n, o in zip(news, olds)])
        rows = cu_q[-1] + c["pad"]
        x = _heads(g, rows, c["hq"] + 2 * c["hk"], c["d"])   # as the projection writes it: queries, keys, values
        s |= {"q": x[:, :c["hq"]], "cu_q": _ints(cu_q), "cu_k": _ints(cu_k) if c["old"] else None}
        if c["old"]:   # the cached tokens' values, and the new ones behind them
            s |= {"k": _heads(g, cu_k[-1], c["hk"], c["d"]), "v": _heads(g, cu_k[-1], c["hk"], c["d"])}
        else:
            s |= {"k": x[:, c["hq"]:c["hq"] + c["hk"]], "v": x[:, c["hq"] + c["hk"]:]}
    elif c["op"] == "prefix":
        lens = _lens(c)
        first, held = -(-c["prefix"] // c["page"]), [-(-n // c["page"]) for n in lens]
        total = first + sum(held) + 2
        ids = _pick(g, total, first + sum(held))
        table = torch.full((c["batch"], max(held) + 1), -1, dtype=torch.int32, device=DEV)
        table[torch.arange(max(held) + 1, device=DEV)[None, :] < _ints(held)[:, None]] = ids[first:]
        s |= {"prefix_len": _ints([c["prefix"]]), "prefix_table": ids[:first].contiguous(), "lens": _ints(lens), "table": table,
              "q": _heads(g, c["batch"], c["hq"], c["d"]),
              "k_pages": _pages(g, total, c["hk"], c["page"], c["d"], c["r"], c["order"]),
              "v_pages": _pages(g, total, c["hk"], c["page"], c["d"], c["r"], c["order"])}
    else:
        m, n = c["tokens"], c["width"]
        weight = lambda: (1 - c["offset"] + 0.2 * torch.randn(n, generator=g, device=DEV)).to(torch.bfloat16)
        h = 3 * torch.randn(m, n, generator=g, device=DEV) * (1 + 5 * (torch.rand(n, generator=g, device=DEV) > 0.99))   # a few channels stand out
        s |= {"y": torch.randn(m, n, generator=g, device=DEV).to(torch.bfloat16), "h": h if c["wide"] else h.to(torch.bfloat16),
              "w_pre": weight(), "w_post": weight() if c["post"] else None, "gate": None}
        if c["gate"] != "none":
            shape = (m, n) if c["gate"] == "token" else (n,)
            s["gate"] = (0.5 + 0.3 * torch.randn(*shape, generator=g, device=DEV)).to(torch.bfloat16)
    return s


# ---- the plain forms -----------------------------------------------------------------------------

def _softmax_sum(x, v):
    """(softmax(x) @ v, log of the exponentials' sum); 0 and -inf for rows of x that are -inf throughout."""
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    return torch.where(total > 0, e @ v / total, 0.0), (top + total.log())[..., 0]


def _capped(x, c):
    return c["cap"] * torch.tanh(x / c["cap"]) if c["cap"] else x


def _plain_prompt(s):
    c = s["c"]
    b, hk, share, d = c["batch"], c["hk"], c["hq"] // c["hk"], c["d"]
    cu_q = s["cu_q"].long()
    cu_k = cu_q if s["cu_k"] is None else s["cu_k"].long()
    nq, nk = cu_q.diff()[:, None], cu_k.diff()[:, None]
    i, j = torch.arange(c["longest"], device=DEV), torch.arange(c["longest"] + c["old"], device=DEV)
    at_q, at_k = (cu_q[:-1, None] + i).clamp(max=len(s["q"]) - 1), (cu_k[:-1, None] + j).clamp(max=len(s["k"]) - 1)
    q = s["q"].float()[at_q].view(b, len(i), hk, share, d).permute(0, 2, 3, 1, 4).reshape(b, hk, share * len(i), d)
    k, v = (s[n].float()[at_k].permute(0, 2, 1, 3) for n in ("k", "v"))
    own_at = (nk - nq + i)[:, :, None]   # a query's own place among the keys
    seen = (j <= own_at) & (i < nq)[:, :, None]
    if c["window"]:
        seen &= j > own_at - c["window"]
    x = _capped(q * d ** -0.5 @ k.transpose(2, 3).contiguous(), c).view(b, hk, share, len(i), len(j))
    x = x.masked_fill_(~seen[:, None, None], -math.inf).view(b, hk, share * len(i), len(j))
    out, lse = _softmax_sum(x, v.contiguous())
    out = out.view(b, hk, share, len(i), d).permute(0, 3, 1, 2, 4).reshape(b, len(i), c["hq"], d)
    lse = lse.view(b, hk, share, len(i)).permute(0, 3, 1, 2).reshape(b, len(i), c["hq"])
    live = i < nq
    got = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device=DEV)
    sums = torch.zeros(s["q"].shape[:2], device=DEV)
    got[at_q[live]], sums[at_q[live]] = out[live].to(torch.bfloat16), lse[live]
    return {"out": got, "lse": sums}


def _values(rows, d, r):
    """What compact cache rows [..., row bytes] stand for, in 32 bits."""
    low = r + (d - r) // 2
    par = rows[..., low:low + 16].contiguous().view(torch.float32)
    b = rows[..., r:low]
    hi = rows[..., :r].float() * par[..., 0:1] + par[..., 1:2]
    lo = torch.stack((b & 15, b >> 4), -1).flatten(-2).float() * par[..., 2:3] + par[..., 3:4]
    return torch.cat((hi, lo), -1)


def _plain_prefix(s):
    c = s["c"]
    b, hk, share, d, page = c["batch"], c["hk"], c["hq"] // c["hk"], c["d"], c["page"]
    n = c["prefix"]
    lens = s["lens"].long()[:, None]
    t, u = torch.arange(n, device=DEV), torch.arange(c["longest"], device=DEV)
    q = s["q"].float().view(b, hk, share, d) * d ** -0.5
    front = s["prefix_table"].long()[t // page]
    kp, vp = (_values(p[front, :, t % page], d, c["r"]).transpose(0, 1).contiguous() for p in (s["k_pages"], s["v_pages"]))
    back = s["table"].long()[:, u // page].clamp(min=0)
    ks, vs = (_values(p[back, :, u % page], d, c["r"]).transpose(1, 2).contiguous() for p in (s["k_pages"], s["v_pages"]))
    xp = _capped(q.permute(1, 0, 2, 3).reshape(hk, b * share, d) @ kp.transpose(1, 2).contiguous(), c)
    xp = xp.view(hk, b, share, n).transpose(0, 1)
    xs = _capped(q @ ks.transpose(2, 3).contiguous(), c)
    seen_p, seen_s = (t < n).expand(b, -1), u < lens
    if c["window"]:
        seen_p, seen_s = t >= n + lens - c["window"], seen_s & (u >= lens - c["window"])
    vs = torch.where((u < lens)[:, None, :, None], vs, 0.0)
    xp, xs = xp.masked_fill(~seen_p[:, None, None], -math.inf), xs.masked_fill(~seen_s[:, None, None], -math.inf)
    top = torch.maximum(xp.amax(-1, keepdim=True), xs.amax(-1, keepdim=True))
    ep, es = torch.exp(xp - top), torch.exp(xs - top)
    total = ep.sum(-1, keepdim=True) + es.sum(-1, keepdim=True)
    front = (ep.transpose(0, 1).reshape(hk, b * share, n) @ vp).view(hk, b, share, d).transpose(0, 1)
    out = (front + es @ vs) / total
    return {"out": out.reshape(b, c["hq"], d).to(torch.bfloat16), "lse": (top + total.log()).view(b, c["hq"])}


def _plain_norm(s):
    c = s["c"]
    scale = lambda x, w: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * (c["offset"] + w.float())
    y = s["y"].float()
    if c["post"]:
        y = scale(y, s["w_post"])
    if s["gate"] is not None:
        y = y * s["gate"].float()
    h = s["h"].float() + c["alpha"] * y
    return {"h": h.to(s["h"].dtype), "x": scale(h, s["w_pre"]).to(torch.bfloat16)}


# ---- one pass ------------------------------------------------------------------------------------

def _own(s):
    from paper_2412_14363_amd import binding as rq
    c, kept = s["c"], s["kept"]  # kept: the buffers that a program which answers request after request has of its own
    if c["op"] == "norm":
        if not kept:
            kept["h"], kept["x"] = torch.empty_like(s["h"]), torch.empty_like(s["y"])
        h, x = rq.resq_norm_residual(s["y"], s["h"], s["w_pre"], w_post=s["w_post"], gate=s["gate"], alpha=c["alpha"], eps=1e-6,
                                     w_offset=c["offset"], h_out=kept["h"], x=kept["x"])
        return {"h": h, "x": x}
    if c["op"] == "prompt":
        if not kept:
            kept["out"] = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device=DEV)   # rows behind the last sequence stay as they are
            kept["lse"] = torch.zeros(s["q"].shape[:2], dtype=torch.float32, device=DEV)
            kept["space"] = rq.resq_attend_prompts_workspace(len(s["q"]), len(s["k"]), c["batch"], c["hq"], c["hk"], c["d"])
        out = rq.resq_attend_prompts(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], scale=c["d"] ** -0.5, softcap=c["cap"], window=c["window"],
                                     out=kept["out"], lse=kept["lse"], workspace=kept["space"])
        return {"out": out, "lse": kept["lse"]}
    if not kept:
        kept["out"] = torch.empty_like(s["q"])
        kept["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEV)
        kept["space"] = rq.resq_attend_kv_prefix_workspace(c["batch"], c["hq"], c["hk"], c["d"])
    out = rq.resq_attend_kv_prefix(s["q"], s["k_pages"], s["v_pages"], s["prefix_len"], s["prefix_table"], s["lens"], s["table"], c["r"],
                                   scale=c["d"] ** -0.5, softcap=c["cap"], window=c["window"], out=kept["out"], lse=kept["lse"],
                                   workspace=kept["space"])
    return {"out": out, "lse": kept["lse"]}


def run(state):
    if own:
        return _own(state)
    return {"prompt": _plain_prompt, "prefix": _plain_prefix, "norm": _plain_norm}[state["c"]["op"]](state)


def _seen(n, window):
    """Keys that queries 0 .. n - 1 see in all: 1, 2, ... up to the window."""
    w = min(n, window) if window else n
    return w * (w + 1) // 2 + (n - w) * w


def work(case):
    c = case
    if c["op"] == "norm":
        m, n = c["tokens"], c["width"]
        gate = {"none": 0, "channel": 2 * n, "token": 2 * m * n}[c["gate"]]
        return {"bytes": m * n * (4 + 2 * (4 if c["wide"] else 2)) + 2 * n * (1 + c["post"]) + gate, "flops": m * n * (10 if c["post"] else 6)}
    if c["op"] == "prompt":
        news, olds = _news(c), _olds(c)
        pairs = sum(_seen(n + o, c["window"]) - _seen(o, c["window"]) for n, o in zip(news, olds))
        rows, keys = sum(news), sum(news) + sum(olds)   # (a window leaves the furthest keys out where old tokens are many)
        if c["window"]:
            keys = sum(min(n + o, n - 1 + c["window"]) for n, o in zip(news, olds) if n)
        return {"bytes": rows * c["hq"] * (4 * c["d"] + 4) + 4 * keys * c["hk"] * c["d"], "flops": 4 * pairs * c["hq"] * c["d"]}
    lens, n, w = _lens(c), c["prefix"], c["window"] or c["prefix"] + c["longest"]
    front = [max(0, min(n, w - k)) for k in lens]
    back = [min(k, w) for k in lens]
    return {"bytes": 2 * (max(front) + sum(back)) * c["hk"] * _row_bytes(c["d"], c["r"]) + c["batch"] * c["hq"] * (4 * c["d"] + 4),
            "flops": 4 * (sum(front) + sum(back)) * c["hq"] * c["d"]}


# ---- from the definitions, in 64 bits -------------------------------------------------------------

def _exact_head(q, k, v, scale, cap, first, last):
    """One head: queries [n, d] over keys first[i] .. last[i] - 1."""
    x = scale * (q @ k.T)
    if cap:
        x = cap * torch.tanh(x / cap)
    t = torch.arange(len(k), device=DEV)
    x[(t < first[:, None]) | (t >= last[:, None])] = -math.inf
    lse = torch.logsumexp(x, 1)
    return torch.exp(x - lse[:, None]) @ v, lse


def _exact_rows(rows, d, r):
    n = r + (d - r) // 2
    words = rows[..., n:n + 16].to(torch.int64).view(*rows.shape[:-1], 4, 4)
    bits = words[..., 0] + (words[..., 1] << 8) + (words[..., 2] << 16) + (words[..., 3] << 24)
    p = bits.to(torch.int32).view(torch.float32).double()
    codes = rows[..., :n].double()
    y = torch.empty(*rows.shape[:-1], d, dtype=torch.float64, device=rows.device)
    y[..., :r] = codes[..., :r] * p[..., 0:1] + p[..., 1:2]
    up = torch.floor(codes[..., r:] / 16)
    y[..., r + 1::2] = up * p[..., 2:3] + p[..., 3:4]
    y[..., r::2] = (codes[..., r:] - 16 * up) * p[..., 2:3] + p[..., 3:4]
    return y


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["op"] == "norm":
        h, y, eps = s["h"].double(), s["y"].double(), 1e-6
        if c["post"]:
            y = y / torch.sqrt((y * y).sum(1, keepdim=True) / c["width"] + eps) * (s["w_post"].double() + c["offset"])
        if s["gate"] is not None:
            y = s["gate"].double() * y
        h = h + y * c["alpha"]
        return {"h": h, "x": h / torch.sqrt((h * h).sum(1, keepdim=True) / c["width"] + eps) * (s["w_pre"].double() + c["offset"])}
    share = c["hq"] // c["hk"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    if c["op"] == "prompt":
        q0 = k0 = 0
        for n, o in zip(_news(c), _olds(c)):
            last = torch.arange(o + 1, o + n + 1, device=DEV)
            first = (last - c["window"]).clamp(min=0) if c["window"] else 0 * last
            for h in range(c["hq"] if n else 0):
                k, v = (s[x][k0:k0 + n + o, h // share].double() for x in ("k", "v"))
                out[q0:q0 + n, h], lse[q0:q0 + n, h] = _exact_head(s["q"][q0:q0 + n, h].double(), k, v, c["d"] ** -0.5, c["cap"], first, last)
            q0, k0 = q0 + n, k0 + n + o
        return {"out": out, "lse": lse}
    n, page = c["prefix"], c["page"]
    for h in range(c["hk"]):
        def values(pages, ids, count):
            return _exact_rows(pages[ids.long(), h].reshape(-1, pages.shape[-1])[:count], c["d"], c["r"])
        front = [values(p, s["prefix_table"], n) for p in (s["k_pages"], s["v_pages"])]
        for b, own_tokens in enumerate(_lens(c)):
            ids = s["table"][b, :-(-own_tokens // page)]
            k, v = (torch.cat((f, values(p, ids, own_tokens))) for f, p in zip(front, (s["k_pages"], s["v_pages"])))
            last = torch.full((share,), n + own_tokens, device=DEV)
            first = (last - c["window"]).clamp(min=0) if c["window"] else 0 * last
            at = slice(h * share, (h + 1) * share)
            out[b, at], lse[b, at] = _exact_head(s["q"][b, at].double(), k, v, c["d"] ** -0.5, c["cap"], first, last)
    return {"out": out, "lse": lse}
