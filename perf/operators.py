"""The operators between a model's query/key/value projections and its output projection when it answers, on this library's
compact K/V cache rows (8-bit and 4-bit codes per head), kept in pages: the plan of a step on the GPU (which page and row
every new token gets), norm and rotation of the query and key heads, the paged writer and reader of the cache, and the
attention of one new token over it.

``run`` computes them from elementary torch operations in 32 bits (64 for angles, and for quotients that are rounded to
codes) where ``own`` is false, and calls ``paper_2412_14363_amd.binding`` where it is true.
"""
import math
import random

import torch

own = False
DEV = "cuda"


# ---- the cases ---------------------------------------------------------------------------------

def listed():
    return [
        # the plan of a generation step: 32 sequences with one new token each
        {"name": "slots_decode_b32", "op": "slots", "batch": 32, "new": 0, "old": 4000, "page": 16, "cap": 32},
        # the plan of a prefill step: 48 prompts of ragged lengths on top of cached prefixes, 16384 new tokens at most
        {"name": "slots_prefill_b48", "op": "slots", "batch": 48, "new": 600, "old": 700, "page": 32, "cap": 16384},
        # one new token of an 8B model: 32 query and 8 key heads, no norm, the smallest rotation
        {"name": "rope_m1", "op": "rope", "tokens": 1, "hq": 32, "hk": 8, "d": 128, "rot": 128, "inter": False, "norm": False,
         "scaling": "none", "far": 8000},
        # the same model on a 2048-token prompt whose positions lie far out, with frequencies stretched for that
        {"name": "rope_m2048_far", "op": "rope", "tokens": 2048, "hq": 32, "hk": 8, "d": 128, "rot": 128, "inter": False,
         "norm": False, "scaling": "banded", "far": 1000000},
        # norm and rotation in one pass, half of each head rotated in the interleaved layout, ragged token count
        {"name": "rope_norm_m5333", "op": "rope", "tokens": 5333, "hq": 14, "hk": 2, "d": 128, "rot": 64, "inter": True,
         "norm": True, "scaling": "linear", "far": 30000},
        # K and V of 64 generating sequences written to their pages, and the values that were written read back
        {"name": "append_m64", "op": "append", "tokens": 64, "heads": 8, "d": 128, "r": 16, "page": 16, "pad": 0, "order": "head"},
        # a ragged prefill batch, the rows behind its last token padding, pages that keep a token's heads together
        {"name": "append_m3001_padded", "op": "append", "tokens": 3001, "heads": 8, "d": 128, "r": 16, "page": 32, "pad": 90,
         "order": "token"},
        # a cached prefix of 16384 tokens back in bf16, for a prefill that attends to it
        {"name": "gather_m16384", "op": "gather", "tokens": 16384, "heads": 8, "d": 128, "r": 16, "page": 16, "pad": 0, "order": "head"},
        # one sequence at a short context: the smallest attention
        {"name": "attend_b1_777", "op": "attend", "batch": 1, "longest": 777, "hq": 32, "hk": 8, "d": 128, "r": 16, "page": 16,
         "order": "head", "window": 0, "cap": 0.0},
        # 48 sequences of ragged lengths, up to 8192 tokens
        {"name": "attend_b48_ragged", "op": "attend", "batch": 48, "longest": 8192, "hq": 32, "hk": 8, "d": 128, "r": 16, "page": 16,
         "order": "head", "window": 0, "cap": 0.0},
        # one long document on a 70B model's heads
        {"name": "attend_b1_131072", "op": "attend", "batch": 1, "longest": 131072, "hq": 64, "hk": 8, "d": 128, "r": 16, "page": 64,
         "order": "head", "window": 0, "cap": 0.0},
        # heads of 64 without sharing, odd pages that keep a token's heads together, a window, capped scores, empty sequences
        {"name": "attend_b24_window_cap", "op": "attend", "batch": 24, "longest": 3500, "hq": 12, "hk": 12, "d": 64, "r": 8, "page": 24,
         "order": "token", "window": 1500, "cap": 30.0},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _group(rng, d):
    return rng.choice([d // 8, d // 8, d // 8, d // 4, 0, d, rng.randrange(0, d + 1, 8)])


def draw(rng):
    op = rng.choice(["slots", "rope", "rope", "append", "gather", "attend", "attend", "attend"])
    order = rng.choice(["head", "head", "token"])
    page = rng.choice([16, 16, 32, 64, 128, 8, 24, rng.randint(1, 100)])
    d = rng.choice([64, 128, 128, 256, 96])
    if op == "slots":
        batch = _log_int(rng, 1, 256)
        new = rng.choice([0, _log_int(rng, 1, 16384 // batch)])
        return {"op": op, "batch": batch, "new": new, "old": _log_int(rng, 1, 8000), "page": max(page, 8),
                "cap": batch if new == 0 else rng.randint(2 * batch * new, 2 * batch * new + 99)}
    if op == "rope":
        inter = rng.random() < 0.5
        rot = rng.choice([d, d, d // 2, d // 4, rng.randrange(2, d + 1, 2)])
        hk = rng.choice([1, 2, 4, 8])
        hq = hk * rng.choice([1, 2, 4, 7])
        return {"op": op, "tokens": _log_int(rng, 1, max(2, 4096 * 40 * 128 // ((hq + hk) * d) // 2)), "hq": hq, "hk": hk, "d": d,
                "rot": rot, "inter": inter, "norm": rng.random() < 0.5, "scaling": rng.choice(["none", "linear", "banded", "ramp"]),
                "far": _log_int(rng, 10, 2000000)}
    if op in ("append", "gather"):
        heads = rng.choice([1, 2, 5, 8, 8, 16])
        tokens = _log_int(rng, 1, (3001 if op == "append" else 16384) * 8 * 128 // (heads * d))
        return {"op": op, "tokens": tokens, "heads": heads, "d": d, "r": _group(rng, d), "page": page,
                "pad": rng.choice([0, 0, rng.randint(1, 50)]), "order": order}
    hk = rng.choice([1, 2, 4, 8, 8, 12])
    share = rng.choice([1, 2, 4, 4, 7, 8, 16, 24])
    batch = _log_int(rng, 1, 64)
    most = 48 * 4096 * 8 * 128 // (batch * hk * d) // 2
    longest = _log_int(rng, 1, max(2, min(131072, most, 1000000000 // (batch * hk * share * d))))
    return {"op": op, "batch": batch, "longest": longest, "hq": hk * share, "hk": hk, "d": d, "r": _group(rng, d), "page": page, "order": order,
            "window": rng.choice([0, 0, _log_int(rng, 1, 8192)]), "cap": rng.choice([0.0, 0.0, 20.0, 50.0])}


# ---- what a case's lengths are (its work goes by them; the seed makes everything else) -----------------------------

def _news(c):
    """Tokens that each request of a plan brings: one each in a generation step, else about `new`, now and then none."""
    rng = random.Random(c["batch"] * 1000003 + c["new"])
    return [1 if c["new"] == 0 else rng.choice([0, c["new"], rng.randint(1, 2 * c["new"])]) for _ in range(c["batch"])]


def _olds(c):
    rng = random.Random(c["batch"] * 1000033 + c["old"])
    return [rng.choice([0, rng.randint(1, 2 * c["old"]), rng.randint(1, 2 * c["old"])]) for _ in range(c["batch"])]


def _lens(c):
    """Cached tokens of each sequence: `longest` for one, ragged below it for the others, some of them without any."""
    rng = random.Random(c["batch"] * 1000037 + c["longest"])
    more = [rng.choice([rng.randint(1, c["longest"])] * 15 + [0]) for _ in range(c["batch"] - 1)]
    at = rng.randint(0, len(more))
    return more[:at] + [c["longest"]] + more[at:]


def _row_bytes(d, r):
    return r + (d - r) // 2 + 16


# ---- inputs ------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pick(g, n, k):
    """k different whole numbers below n, in any order."""
    return torch.randperm(n, generator=g, device=DEV)[:k].to(torch.int32)


def _heads(g, *shape, r=0):
    """bf16 head vectors; the first r channels, the ones that are kept in 8 bits, vary most."""
    x = torch.randn(*shape, generator=g, device=DEV)
    x += 0.3 * torch.randn(shape[-1], generator=g, device=DEV)
    x[..., :r] *= 5.0
    return x.to(torch.bfloat16)


def _pages(g, n, heads, page, d, r, order, filled):
    """Cache pages [n, heads, page, row bytes], in memory in that order or with a token's heads together; filled with
    quantized heads or with zeros."""
    nb = _row_bytes(d, r)
    if filled:
        rows = _as_rows(_heads(g, n, heads, page, d, r=r), r)
    else:
        rows = torch.zeros(n, heads, page, nb, dtype=torch.uint8, device=DEV)
    return rows.transpose(1, 2).contiguous().transpose(1, 2) if order == "token" else rows


def _frequencies(c):
    """Angle per position of each pair of channels, in 64 bits: the geometric row, as it is or stretched for long contexts
    (all alike; by bands of wavelengths; by a ramp over the pairs)."""
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device=DEV)
    f = 500000.0 ** (-2.0 * i / c["rot"])
    if c["scaling"] == "linear":
        return f / 4.0
    if c["scaling"] == "banded":
        turns = 8192.0 * f / (2.0 * math.pi)
        return torch.lerp(f / 8.0, f, ((turns - 1.0) / 3.0).clamp(0.0, 1.0))
    if c["scaling"] == "ramp":
        return torch.lerp(f, f / 16.0, (i / max(1, len(i) - 1)).clamp(0.0, 1.0))
    return f


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    s = {"c": c, "kept": {}}
    if c["op"] == "slots":
        new, old = _news(c), _olds(c)
        have = [-(-o // c["page"]) for o in old]
        need = [-(-(o + n) // c["page"]) for o, n in zip(old, new)]
        total = 2 * sum(need) + 8
        ids = _pick(g, total, total)
        width = max(need) + 3
        table = torch.full((c["batch"], width), -1, dtype=torch.int32, device=DEV)
        held = torch.arange(width, device=DEV)[None, :] < _ints(have)[:, None]
        table[held] = ids[:sum(have)]
        s |= {"lens": _ints(old), "new": _ints(new), "free": ids[sum(have):].contiguous(), "table": table, "pages": total,
              "taken": _ints([3])}
    elif c["op"] == "rope":
        x = _heads(g, c["tokens"], c["hq"] + 2 * c["hk"], c["d"])  # as the projection writes it: queries, keys, values
        s |= {"x": x[:, :c["hq"] + c["hk"]], "freq": _frequencies(c), "mscale": 1.1 if c["scaling"] == "ramp" else 1.0,
              "pos": torch.randint(0, c["far"], (c["tokens"],), generator=g, device=DEV, dtype=torch.int32),
              "wq": (1 + 0.2 * torch.randn(c["d"], generator=g, device=DEV)).to(torch.bfloat16) if c["norm"] else None,
              "wk": (1 + 0.2 * torch.randn(c["d"], generator=g, device=DEV)).to(torch.bfloat16) if c["norm"] else None}
    elif c["op"] in ("append", "gather"):
        t, h, d, r = c["tokens"], c["heads"], c["d"], c["r"]
        n = -(-t // c["page"]) + 2
        slots = _pick(g, n * c["page"], t)
        if c["pad"]:
            slots[max(1, t - c["pad"]):] = -1
        s |= {"slots": slots, "k_pages": _pages(g, n, h, c["page"], d, r, c["order"], c["op"] == "gather"),
              "v_pages": _pages(g, n, h, c["page"], d, r, c["order"], c["op"] == "gather")}
        if c["op"] == "append":
            s |= {"k": _heads(g, t, h, d, r=r), "v": _heads(g, t, h, d, r=r)}
    else:
        lens = _lens(c)
        held = [-(-n // c["page"]) for n in lens]
        total = sum(held) + 2
        table = torch.full((c["batch"], max(held) + 1), -1, dtype=torch.int32, device=DEV)
        table[torch.arange(max(held) + 1, device=DEV)[None, :] < _ints(held)[:, None]] = _pick(g, total, sum(held))
        s |= {"lens": _ints(lens), "table": table, "q": _heads(g, c["batch"], c["hq"], c["d"]),
              "k_pages": _pages(g, total, c["hk"], c["page"], c["d"], c["r"], c["order"], True),
              "v_pages": _pages(g, total, c["hk"], c["page"], c["d"], c["r"], c["order"], True),
              "lse": torch.empty(c["batch"], c["hq"], dtype=torch.float32, device=DEV),
              "scale": c["d"] ** -0.5}
    return s


# ---- the plain forms -----------------------------------------------------------------------------

def _quantize(x, levels):
    """Codes, scale and zero-point of each row of x: Eq. 1's asymmetric branch, differences and quotients rounded to 32
    bits (taken in 64, so that every one of them is the correctly rounded one)."""
    z = x.amin(-1, keepdim=True)
    span = (x.amax(-1, keepdim=True) - z)
    scale = torch.where(span == 0, 1.0, (span.double() / levels).float())
    return ((x - z).double() / scale.double()).float().round().clamp(0, levels), scale, z


def _parts(x, r):
    """(codes, scale, zero) of the 8-bit and the 4-bit channels of bf16 rows x; an absent group is None."""
    x = x.float()
    return (_quantize(x[..., :r], 255) if r else None), (_quantize(x[..., r:], 15) if r < x.shape[-1] else None)


def _as_rows(x, r):
    """Compact cache rows: 8-bit codes, pairs of 4-bit codes, then both groups' scale and zero-point."""
    hi, lo = _parts(x, r)
    one = torch.ones(*x.shape[:-1], 1, device=x.device)
    got = [hi[0].to(torch.uint8)] if hi else []
    if lo:
        q = lo[0].to(torch.uint8)
        got.append(q[..., 0::2] | (q[..., 1::2] << 4))
    par = torch.cat(list(hi[1:] if hi else (one, 0 * one)) + list(lo[1:] if lo else (one, 0 * one)), -1)
    return torch.cat(got + [par.contiguous().view(torch.uint8)], -1)


def _values(rows, d, r):
    """What compact cache rows [..., row bytes] stand for, in 32 bits."""
    low = r + (d - r) // 2
    par = rows[..., low:low + 16].contiguous().view(torch.float32)
    b = rows[..., r:low]
    hi = rows[..., :r].float() * par[..., 0:1] + par[..., 1:2]
    lo = torch.stack((b & 15, b >> 4), -1).flatten(-2).float() * par[..., 2:3] + par[..., 3:4]
    return torch.cat((hi, lo), -1)


def _plain_slots(s):
    c = s["c"]
    page, cap, width = c["page"], c["cap"], s["table"].shape[1]
    lens, new = s["lens"].long(), s["new"].long()
    have = (lens + page - 1) // page
    need = (lens + new + page - 1) // page - have
    zero = torch.zeros(1, dtype=torch.int64, device=DEV)
    cu, cp = torch.cat((zero, new.cumsum(0))), torch.cat((zero, need.cumsum(0)))
    taken = s["taken"].long()[0]
    state = torch.where(((lens < 0) | (new < 0)).any(), 4, torch.where(
        cu[-1] > cap, 3, torch.where(((have + need) > width).any(), 2, torch.where(taken + cp[-1] > s["free"].numel(), 1, 0))))
    good = state == 0
    t = torch.arange(cap, device=DEV)
    b = torch.searchsorted(cu[1:], t, right=True).clamp(max=c["batch"] - 1)
    live = (t < cu[-1]) & good
    pos = torch.where(live, lens[b] + t - cu[b], 0)
    at = pos // page
    fresh = live & (at >= have[b])
    got = s["free"].long()[(taken + cp[b] + at - have[b]).clamp(0, s["free"].numel() - 1)]
    wide = torch.cat((s["table"], torch.full_like(s["table"][:, :1], -1)), 1).long()
    ids = torch.where(fresh, got, wide[b, at.clamp(max=width)])
    wide[b, torch.where(fresh, at, width)] = torch.where(fresh, got, -1)
    i32 = torch.int32
    return {"lens": torch.where(good, lens + new, lens).to(i32), "cu_tokens": torch.where(good, cu, 0).to(i32),
            "cu_pages": torch.where(good, cp, 0).to(i32), "positions": pos.to(i32),
            "slots": torch.where(live, ids * page + pos % page, -1).to(i32), "table": wide[:, :width].to(i32),
            "state": torch.stack((torch.where(good, taken + cp[-1], taken), state)).to(i32)}


def _plain_rope(s):
    c, x = s["c"], s["x"].float()
    if c["norm"]:
        w = torch.cat((s["wq"].float().expand(c["hq"], -1), s["wk"].float().expand(c["hk"], -1)))
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
    angle = s["pos"].double()[:, None, None] * s["freq"]
    cos, sin = (s["mscale"] * angle.cos()).float(), (s["mscale"] * angle.sin()).float()
    rot = x[..., :c["rot"]]
    a, b = (rot[..., 0::2], rot[..., 1::2]) if c["inter"] else rot.chunk(2, -1)
    turned = (a * cos - b * sin, b * cos + a * sin)
    turned = torch.stack(turned, -1).flatten(-2) if c["inter"] else torch.cat(turned, -1)
    return torch.cat((turned, x[..., c["rot"]:]), -1).to(torch.bfloat16)


def _plain_append(s):
    c, got = s["c"], []
    live = (s["slots"] >= 0)[:, None, None]
    for x in (s["k"], s["v"]):
        hi, lo = _parts(x, c["r"])
        y = torch.cat([q * scale + z for q, scale, z in (p for p in (hi, lo) if p)], -1)
        got.append(torch.where(live, y, 0.0).to(torch.bfloat16))
    return got


def _rows_at(pages, slots, page):
    """Rows [..., heads, row bytes] of the tokens in `slots`."""
    at = slots.long().clamp(min=0)
    return pages[at // page, :, at % page]


def _plain_gather(s):
    c = s["c"]
    live = (s["slots"] >= 0)[:, None, None]
    return [torch.where(live, _values(_rows_at(p, s["slots"], c["page"]), c["d"], c["r"]), 0.0).to(torch.bfloat16)
            for p in (s["k_pages"], s["v_pages"])]


def _plain_attend(s):
    c = s["c"]
    b, hk, d, page = c["batch"], c["hk"], c["d"], c["page"]
    t = torch.arange(c["longest"], device=DEV)
    lens = s["lens"].long()[:, None]
    seen = t < lens
    if c["window"]:
        seen = seen & (t >= lens - c["window"])
    slots = s["table"].long()[:, t // page] * page + t % page
    k, v = (_values(_rows_at(p, slots, page), d, c["r"]).transpose(1, 2) for p in (s["k_pages"], s["v_pages"]))
    x = s["q"].float().view(b, hk, c["hq"] // hk, d) * s["scale"] @ k.transpose(2, 3).contiguous()
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    x = x.masked_fill(~seen[:, None, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    v = torch.where(seen[:, None, :, None], v, 0.0)
    out = torch.where(total > 0, e @ v / total, 0.0)
    return {"out": out.view(b, c["hq"], d).to(torch.bfloat16), "lse": (top + total.log()).view(b, c["hq"])}


# ---- one pass ------------------------------------------------------------------------------------

def _own(s):
    from paper_2412_14363_amd import binding as rq
    c, kept = s["c"], s["kept"]  # kept: the buffers that a program which answers token after token has of its own
    if c["op"] == "slots":
        if not kept:
            kept["plan"] = rq.KvSlots(c["batch"], c["cap"])
        p = rq.resq_kv_slots(s["lens"], s["new"], s["free"], s["taken"], s["table"], c["page"], s["pages"], out=kept["plan"])
        return {"lens": p.lens, "cu_tokens": p.cu_tokens, "cu_pages": p.cu_pages, "positions": p.positions, "slots": p.slots,
                "table": s["table"], "state": p.state}
    if c["op"] == "rope":
        if not kept:
            kept["y"] = torch.empty(s["x"].shape, dtype=torch.bfloat16, device=DEV)
        return rq.resq_rope_heads(s["x"], s["pos"], s["freq"], heads_q=c["hq"], w_q=s["wq"], w_k=s["wk"], eps=1e-6,
                                  interleaved=c["inter"], mscale=s["mscale"], out=kept["y"])
    if c["op"] in ("append", "gather"):
        if not kept:
            kept["k"], kept["v"] = (torch.empty(c["tokens"], c["heads"], c["d"], dtype=torch.bfloat16, device=DEV) for _ in range(2))
        if c["op"] == "append":
            rq.resq_append_kv_cache(s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"], c["r"])
        return list(rq.resq_gather_kv_cache(s["k_pages"], s["v_pages"], s["slots"], c["r"], k=kept["k"], v=kept["v"]))
    if not kept:
        kept["out"] = torch.empty_like(s["q"])
        kept["space"] = rq.resq_attend_kv_cache_workspace(c["batch"], c["hq"], c["hk"], c["d"])
    out = rq.resq_attend_kv_cache(s["q"], s["k_pages"], s["v_pages"], s["lens"], s["table"], c["r"], scale=s["scale"],
                                  softcap=c["cap"], window=c["window"], out=kept["out"], lse=s["lse"], workspace=kept["space"])
    return {"out": out, "lse": s["lse"]}


def run(state):
    if own:
        return _own(state)
    return {"slots": _plain_slots, "rope": _plain_rope, "append": _plain_append, "gather": _plain_gather,
            "attend": _plain_attend}[state["c"]["op"]](state)


def work(case):
    c = case
    if c["op"] == "slots":  # lengths and counts in and out, a position and a slot per token, a table entry and a page per page
        new, old = _news(c), _olds(c)
        fresh = sum(-(-(o + n) // c["page"]) - -(-o // c["page"]) for o, n in zip(old, new))
        return {"bytes": 4 * (5 * c["batch"] + 2 * c["cap"] + 2 * fresh), "flops": 4 * c["cap"]}
    if c["op"] == "rope":
        n = c["tokens"] * (c["hq"] + c["hk"])
        return {"bytes": 4 * n * c["d"] + 4 * c["tokens"] + 4 * c["rot"], "flops": n * (3 * c["rot"] + (4 * c["d"] if c["norm"] else 0))}
    nb = _row_bytes(c["d"], c["r"])
    if c["op"] in ("append", "gather"):
        t = max(1, c["tokens"] - c["pad"]) if c["pad"] else c["tokens"]
        rows, every = 2 * t * c["heads"], 2 * c["tokens"] * c["heads"]
        wrote = rows * (2 * c["d"] + nb) if c["op"] == "append" else 0
        return {"bytes": wrote + rows * nb + every * 2 * c["d"] + 4 * c["tokens"], "flops": (12 if wrote else 2) * rows * c["d"]}
    seen = sum(min(n, c["window"]) if c["window"] else n for n in _lens(c))
    return {"bytes": 2 * seen * c["hk"] * nb + 4 * c["batch"] * c["hq"] * (c["d"] + 1) + 4 * sum(-(-n // c["page"]) for n in _lens(c)),
            "flops": 4 * seen * c["hq"] * c["d"]}


# ---- from the definitions, in 64 bits -------------------------------------------------------------

def _exact_codes(x, levels):
    """The value that the quantizer leaves of each element: its definition rounds the span's quotient, the difference and
    the quotient to 32 bits, and those roundings are part of it."""
    low, high = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
    step = ((high - low).float().double() / levels).float().double()
    step[step == 0] = 1.0
    q = torch.round(((x - low).float().double() / step).float().double())
    return q.clamp(0, levels) * step + low


def _exact_row(rows, d, r):
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
    if c["op"] == "slots":  # whole numbers alone
        return None
    if c["op"] == "rope":
        x = s["x"].double()
        if c["norm"]:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["d"] + 1e-6)
            x[:, :c["hq"]] *= s["wq"].double()
            x[:, c["hq"]:] *= s["wk"].double()
        y, half = x.clone(), c["rot"] // 2
        for i in range(half):
            m, n = (2 * i, 2 * i + 1) if c["inter"] else (i, i + half)
            turn = s["mscale"] * torch.exp(1j * (s["pos"].double() * s["freq"][i]))[:, None] * torch.complex(x[..., m], x[..., n])
            y[..., m], y[..., n] = turn.real, turn.imag
        return y
    d, r = c["d"], c["r"]
    if c["op"] == "append":
        got = []
        for x in (s["k"].double(), s["v"].double()):
            y = x.clone()
            if r:
                y[..., :r] = _exact_codes(x[..., :r], 255)
            if r < d:
                y[..., r:] = _exact_codes(x[..., r:], 15)
            y[s["slots"] < 0] = 0
            got.append(y)
        return got
    if c["op"] == "gather":
        got = []
        for p in (s["k_pages"], s["v_pages"]):
            flat = p.permute(0, 2, 1, 3).reshape(-1, c["heads"], p.shape[-1])
            y = torch.zeros(c["tokens"], c["heads"], d, dtype=torch.float64, device=DEV)
            live = s["slots"] >= 0
            y[live] = _exact_row(flat[s["slots"][live].long()], d, r)
            got.append(y)
        return got
    out = torch.zeros(c["batch"], c["hq"], d, dtype=torch.float64, device=DEV)
    lse = torch.full((c["batch"], c["hq"]), -math.inf, dtype=torch.float64, device=DEV)
    share = c["hq"] // c["hk"]
    for b, n in enumerate(_lens(c)):
        first = max(0, n - c["window"]) if c["window"] else 0
        if n == 0:
            continue
        ids = s["table"][b, :-(-n // c["page"])].long()
        for h in range(c["hk"]):
            k, v = (_exact_row(p[ids, h].reshape(-1, p.shape[-1])[first:n], d, r) for p in (s["k_pages"], s["v_pages"]))
            for i in range(h * share, (h + 1) * share):
                x = (k * s["q"][b, i].double()).sum(-1) * s["scale"]
                if c["cap"]:
                    x = c["cap"] * torch.tanh(x / c["cap"])
                lse[b, i] = torch.logsumexp(x, 0)
                out[b, i] = (torch.exp(x - lse[b, i])[:, None] * v).sum(0)
    return {"out": out, "lse": lse}
