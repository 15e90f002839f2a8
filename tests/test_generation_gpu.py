"""The operators of a generation step on the GPU (plan, position embedding, paged cache, attention) against plain 64-bit
implementations (generation_util.py) and, where the library has the same arithmetic already, bit for bit against that."""
import itertools
import math
from decimal import Decimal, getcontext

import pytest
import torch

import generation_util as plain

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def rq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU; there is no CPU fallback")
    from paper_2412_14363_amd import binding
    binding.lib()
    return binding


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ---- the plan ----------------------------------------------------------------------------------

def plan_inputs(seed, batch, new, old, page, width_pad=2, cap_pad=5):
    g = gen(seed)
    lens = torch.randint(0, old + 1, (batch,), generator=g).tolist()
    news = torch.randint(0, new + 1, (batch,), generator=g).tolist()
    held = [-(-n // page) for n in lens]
    want = [-(-(n + a) // page) for n, a in zip(lens, news)]
    total = sum(want) + 7
    ids = torch.randperm(total, generator=g).tolist()
    width = max(want) + width_pad
    table, at = [], 0
    for h in held:
        table.append(ids[at:at + h] + [-1] * (width - h))
        at += h
    return lens, news, ids[at:], table, total, max(1, sum(news) + cap_pad)


def run_plan(rq, lens, news, free, taken, table, page, num_pages, cap, out=None):
    t = ints(table)
    p = rq.resq_kv_slots(ints(lens), ints(news), ints(free), ints([taken]), t, page, num_pages, out=out, max_tokens=cap)
    torch.cuda.synchronize()
    return [x.tolist() for x in (p.lens, p.cu_tokens, p.cu_pages, p.positions, p.slots, t, p.state)]


@pytest.mark.parametrize("batch,new,old,page,cap_pad", [
    (1, 1, 0, 16, 0), (1, 1, 100, 1, 0), (3, 40, 33, 16, 0), (17, 5, 1000, 24, 300), (64, 1, 4000, 16, 0), (255, 3, 70, 7, 1000),
    (1024, 1, 50, 16, 0), (1025, 2, 20, 16, 9), (5000, 1, 9, 4, 0), (4, 5000, 3000, 64, 1), (2, 40000, 10, 128, 4096), (9, 0, 30, 16, 3)])
def test_plan(rq, batch, new, old, page, cap_pad):
    lens, news, free, table, total, cap = plan_inputs(batch + new, batch, new, old, page, cap_pad=cap_pad)
    got = run_plan(rq, lens, news, free, 2, table, page, total, cap)
    assert got == list(map(lambda x: [list(r) for r in x] if x and isinstance(x[0], list) else list(x),
                           plain.plan(lens, news, free, 2, table, page, total, cap)))


@pytest.mark.parametrize("fault,status", [("pages", 1), ("width", 2), ("cap", 3), ("len", 4), ("new", 4), ("taken", 4), ("cap+len", 4)])
def test_plan_refuses_as_a_whole(rq, fault, status):
    lens, news, free, table, total, cap = plan_inputs(3, 20, 30, 200, 16)
    taken = 0
    if fault == "pages":
        free = free[:sum(-(-(n + a) // 16) - -(-n // 16) for n, a in zip(lens, news)) - 1]
    if fault == "width":
        width = max(-(-(n + a) // 16) for n, a in zip(lens, news)) - 1
        table = [t[:width] for t in table]
    if "cap" in fault:
        cap = sum(news) - 1
    if "len" in fault:
        lens[7] = -1
    if fault == "new":
        news[19] = -5
    if fault == "taken":
        taken = -1
    got = run_plan(rq, lens, news, free, taken, table, 16, total, cap)
    assert got == [list(x) for x in plain.plan(lens, news, free, taken, table, 16, total, cap)]
    assert got[6] == [taken, status] and set(got[4]) == {-1} and got[0] == lens


def test_plan_sums_do_not_wrap(rq):
    # 65536 requests of 2^16 new tokens each: 2^32 in all, more than max_tokens, and 0 modulo 2^32
    n = 65536
    t = torch.zeros(n, 8, dtype=torch.int32, device=DEV)
    p = rq.resq_kv_slots(torch.zeros(n, dtype=torch.int32, device=DEV), torch.full((n,), 1 << 16, dtype=torch.int32, device=DEV),
                         ints([1, 2, 3]), ints([0]), t, 1 << 20, 100, max_tokens=10)
    assert p.state.tolist() == [0, 3] and p.slots.tolist() == [-1] * 10 and not t.any()


def test_plan_goes_on_from_its_own_state(rq):
    # in place, step after step, as a captured step does it: lens and taken are the outputs of the step before
    page, batch = 4, 5
    free, width, total = list(range(60, 0, -1)), 20, 64
    table = [[-1] * width for _ in range(batch)]
    lens, taken = [0] * batch, 0
    t, p = ints(table), rq.KvSlots(batch, 16)
    news = ints([0] * batch)
    for step in range(12):
        add = [(step + b) % 4 for b in range(batch)]
        news.copy_(ints(add))
        rq.resq_kv_slots(p.lens, news, ints(free), None, t, page, total, out=p)
        lens, cu, cp, pos, slots, table, (taken, status) = plain.plan(lens, add, free, taken, table, page, total, 16)
        assert status == 0 and p.state.tolist() == [taken, 0]
        assert (p.lens.tolist(), p.cu_tokens.tolist(), p.cu_pages.tolist()) == (lens, cu, cp)
        assert (p.positions.tolist(), p.slots.tolist(), t.tolist()) == (pos, slots, table)


@pytest.mark.parametrize("batch,cap,new", [(1, 1025, 600), (7, 3000, 300), (700, 1400, 2), (4096, 1024, 0), (4097, 900, 0), (5000, 6000, 1)])
@pytest.mark.parametrize("own", ["lens and taken", "lens", "taken"])
def test_plan_in_place_by_one_launch_and_by_two(rq, batch, cap, new, own):
    """More than 1024 tokens, or 4096 requests, in place: two steps, a refusal in between that changes nothing."""
    g = gen(batch + cap)
    page, width = 16, 80
    total = batch * 4 + 200
    free, table = torch.randperm(total, generator=g).tolist(), [[-1] * width for _ in range(batch)]
    t, p, lens, taken = ints(table), rq.KvSlots(batch, cap), [0] * batch, 0
    free_pages = ints(free)
    for step in range(3):
        add = torch.randint(0, new + 1, (batch,), generator=g).tolist()
        if new == 0:
            for b in torch.randint(0, batch, (40,), generator=g).tolist():
                add[b] = 20
        if step == 1:
            add[batch // 2] = cap + 1
        a = p.lens if "lens" in own else ints(lens)
        b = None if "taken" in own else ints([taken])
        rq.resq_kv_slots(a, ints(add), free_pages, b, t, page, total, out=p)
        lens, cu, cp, positions, slots, table, state = plain.plan(lens, add, free, taken, table, page, total, cap)
        assert state[1] == (3 if step == 1 else 0)
        assert (p.state.tolist(), p.lens.tolist(), p.cu_tokens.tolist(), p.cu_pages.tolist()) == (state, lens, list(cu), list(cp))
        assert (p.positions.tolist(), p.slots.tolist(), t.tolist()) == (list(positions), list(slots), [list(x) for x in table])
        taken = state[0]


def test_plan_on_another_stream(rq):
    # buffers that the call makes for itself are cleared before the plan is in them, whatever the current stream still does
    side, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device=DEV)
    args = [ints([5, 0, 16]), ints([1, 3, 2]), ints([7, 4, 2, 9])]
    table, taken = ints([[3, -1], [-1, -1], [1, -1]]), ints([0])
    torch.cuda.synchronize()
    for _ in range(20):
        busy = busy @ busy * 1e-2
    p = rq.resq_kv_slots(*args, taken, table, 16, 10, max_tokens=8, stream=side)
    torch.cuda.synchronize()
    assert p.slots.tolist() == [3 * 16 + 5, 7 * 16, 7 * 16 + 1, 7 * 16 + 2, 4 * 16, 4 * 16 + 1, -1, -1]
    assert p.positions.tolist() == [5, 0, 1, 2, 16, 17, 0, 0] and p.state.tolist() == [2, 0] and p.lens.tolist() == [6, 3, 18]


def test_plan_leaves_out_pages_that_do_not_exist(rq):
    # a table entry and a free page outside [0, num_pages): their tokens get no slot
    table = [[99, -1, -1], [1, -1, -1]]
    got = run_plan(rq, [3, 2], [3, 9], [77, 2, -3], 0, table, 4, 5, 12)
    want = plain.plan([3, 2], [3, 9], [77, 2, -3], 0, table, 4, 5, 12)
    assert got == [list(x) for x in want]
    assert got[4][:12] == [-1, -1, -1, 6, 7, 8, 9, 10, 11, -1, -1, -1]


# ---- norm and rotation --------------------------------------------------------------------------

def check_rope(rq, x, positions, freq, heads_q, w_q, w_k, interleaved, mscale, out=None, eps=1e-6):
    before = x.clone()
    y = rq.resq_rope_heads(x, positions, freq, heads_q=heads_q, w_q=w_q, w_k=w_k, eps=eps, interleaved=interleaved, mscale=mscale, out=out)
    torch.cuda.synchronize()
    want, size = plain.rope(before, positions, freq, heads_q, w_q, w_k, eps, interleaved, mscale)
    # a rounding to bf16, half of torch.finfo(bfloat16).eps; before it in fp32 a sum of d squares (at most 24 roundings on
    # the way of each term), a root, a quotient, the products, and angles good to 2^-21: 2^-18 of the operands' size
    off = (y.cpu().double() - want).abs()
    bad = off > 2.0 ** -8 * want.abs() + 2.0 ** -18 * size + 1e-38
    assert not bad.any(), (int(bad.sum()), float((off / (size + 1e-30)).max()))
    return y


@pytest.mark.parametrize("d,rot", [(128, 128), (128, 64), (64, 64), (256, 256), (96, 96), (80, 32), (512, 512), (128, 0), (64, 10), (34, 34),
                                   (2, 2), (128, 16), (200, 8), (72, 24)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_rope(rq, d, rot, interleaved, norm):
    for tokens, hq, hk in ((1, 4, 1), (37, 3, 2), (5, 0, 2), (6, 7, 0), (130, 32, 8)):
        g = gen(tokens * d + rot)
        x = torch.randn(tokens, hq + hk, d, generator=g).to(torch.bfloat16).to(DEV)
        w = [(1 + 0.3 * torch.randn(d, generator=g)).to(torch.bfloat16).to(DEV) for _ in range(2)] if norm else [None, None]
        pos = torch.randint(0, 100000, (tokens,), generator=g, dtype=torch.int32).to(DEV)
        freq = rq.resq_rope_frequencies(rot, base=500000.0)[0] if rot else None
        check_rope(rq, x, pos, freq, hq, w[0], w[1], interleaved, 1.25)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_at_far_positions(rq, interleaved):
    # the angle of the fastest pair at 2^31 - 1 is 2^31 radians: in fp32 nothing of it would be left
    x = torch.randn(9, 3, 64, generator=gen(1)).to(torch.bfloat16).to(DEV)
    pos = ints([0, 1, -1, 1 << 20, (1 << 24) + 1, 2147483647, -2147483648, 1234567891, 31415926])
    check_rope(rq, x, pos, rq.resq_rope_frequencies(64)[0], 2, None, None, interleaved, 1.0)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(128, 54), (128, 102), (96, 24), (64, 22), (64, 6), (256, 250), (512, 500), (512, 510), (10, 4), (2, 2), (90, 90)])
def test_rope_of_any_width(rq, d, rot, interleaved):
    # widths that cut pieces of eight channels anywhere, many tokens to a workgroup and one, with values beside the turned channels that
    # must reach no other channel
    g = gen(d + rot)
    freq, _ = rq.resq_rope_frequencies(rot)
    w = (1 + 0.2 * torch.randn(d, generator=g)).to(torch.bfloat16).to(DEV)
    for tokens, heads in ((1, 3), (37, 5), (2100, 3)):
        x = torch.randn(tokens, heads, d, generator=g).to(torch.bfloat16).to(DEV)
        pos = torch.randint(0, 5000, (tokens,), generator=g).to(torch.int32).to(DEV)
        check_rope(rq, x, pos, freq, 2, w, w, interleaved, 1.25)
        inplace = x.clone()
        assert torch.equal(rq.resq_rope_heads(inplace, pos, freq, interleaved=interleaved, out=inplace),
                           check_rope(rq, x, pos, freq, heads, None, None, interleaved, 1.0))
        if rot < d:
            x[..., rot] = float("inf")
            out = rq.resq_rope_heads(x, pos, freq, interleaved=interleaved)
            assert bool((out[..., rot] == float("inf")).all()) and int(out.isfinite().sum()) == tokens * heads * (d - 1)


@pytest.mark.parametrize("d,rot", [(128, 128), (96, 40), (66, 66)])
@pytest.mark.parametrize("interleaved,norm", [(False, True), (True, False)])
def test_rope_layouts(rq, d, rot, interleaved, norm):
    # heads of a wider projection, head-major memory, broadcast input, unaligned rows, in place: the rest of each buffer stays
    g = gen(d)
    freq, mscale = rq.resq_rope_frequencies(rot, scaling="ramp", factor=8.0, low=1.0, high=32.0, original_len=4096)
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(torch.bfloat16).to(DEV) for _ in range(2)] if norm else [None, None]
    tokens, heads = 21, 6
    pos = torch.randint(0, 30000, (tokens,), generator=g, dtype=torch.int32).to(DEV)
    for shift, order in itertools.product((0, 1, 8), ("token", "head", "same", "expand")):
        width = 9 * d + shift
        flat = torch.randn(tokens, width, generator=g).to(torch.bfloat16).to(DEV)
        x = flat[:, shift:shift + heads * d].unflatten(1, (heads, d))
        buf = torch.full((heads, tokens, d + shift), 7.0, dtype=torch.bfloat16, device=DEV)
        if order == "token":
            y = check_rope(rq, x, pos, freq, 4, *w, interleaved, mscale)
            assert y.is_contiguous()
        elif order == "head":
            check_rope(rq, x, pos, freq, 4, *w, interleaved, mscale, out=buf.transpose(0, 1)[..., shift:])
            assert bool((buf[..., :shift] == 7).all())
        elif order == "same":
            keep = flat.clone()
            check_rope(rq, x, pos, freq, 4, *w, interleaved, mscale, out=x)
            assert torch.equal(flat[:, :shift], keep[:, :shift]) and torch.equal(flat[:, shift + heads * d:], keep[:, shift + heads * d:])
        else:
            check_rope(rq, x[:, :1].expand(-1, heads, -1), pos, freq, 4, *w, interleaved, mscale)


def test_rope_angles_near_whole_turns(rq):
    """(1, 0) turned by an angle that is a tiny rest of many turns: its sine is that rest, in fp32 (2^-22 for the rounding, the sine and the
    products) and rounded to bf16, however far the position."""
    getcontext().prec = 90
    turn = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")
    freq = torch.tensor([1.0, 500000.0 ** (-2 / 128), 0.7071, 0.0123456789], dtype=torch.float64)
    g = torch.Generator().manual_seed(8)
    near = torch.randint(1 << 29, (1 << 31) - 1, (1 << 20,), generator=g).double()
    positions = [0, 1, 710, 312689, 4272943, 411557987, 2147483647, -411557987]
    for f in freq:   # the nearest of a million far positions
        rest = near * (f / (2 * math.pi))
        positions.append(int(near[(rest - rest.round()).abs().argmin()]))
    x = torch.zeros(len(positions), 1, 8)
    x[..., :4] = 1
    y = rq.resq_rope_heads(x.to(torch.bfloat16).to(DEV), ints(positions), freq.to(DEV)).cpu().double()
    for t, p in enumerate(positions):
        for i, f in enumerate(freq.tolist()):
            angle = p * Decimal(f)
            want = math.sin(float(angle - turn * (angle / turn).to_integral_value()))
            assert abs(float(y[t, 0, 4 + i]) - want) <= (2.0 ** -8 + 2.0 ** -21) * abs(want), (p, f, want, float(y[t, 0, 4 + i]))


def test_rope_of_zeros_huge_and_no_tokens(rq):
    freq = rq.resq_rope_frequencies(64)[0]
    w = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device=DEV)
    x[1] = 1e18   # the sum of 64 squares is below the largest fp32
    x[1, :, 1::2] = -1e17
    check_rope(rq, x, ints([5, 6, 7]), freq, 1, w, w, False, 1.0)
    assert rq.resq_rope_heads(x[:0], ints([]), freq).shape == (0, 2, 64)


# ---- writer and reader ---------------------------------------------------------------------------

@pytest.mark.parametrize("d,r", [(128, 16), (64, 8), (256, 32), (512, 64), (128, 0), (128, 128), (8, 0), (8, 8), (72, 24), (264, 8)])
@pytest.mark.parametrize("order", ["head", "token"])
def test_append_and_gather(rq, d, r, order):
    nb = plain.row_bytes(d, r)
    for tokens, heads, page, pad in ((1, 1, 1, 0), (5, 3, 16, 4), (67, 8, 24, 0), (300, 2, 7, 12)):
        g = gen(tokens + d + r)
        pages = -(-tokens // page) + 3
        wide = torch.randn(tokens, 2 * heads, d + 8, generator=g).to(torch.bfloat16).to(DEV)
        wide[0] = 2.5                                   # a constant head: scale 1
        k, v = wide[:, :heads, :d], wide[:, heads:, :d]
        buf = [plain.make_pages(g, pages, heads, page, d, r, order, pad) for _ in range(2)]
        was = [b.clone() for b in buf]
        slots = torch.randperm(pages * page, generator=g)[:tokens].to(torch.int32)
        slots[tokens // 2:tokens // 2 + 3] = torch.tensor([-1, pages * page, -2147483648][:max(0, min(3, tokens - tokens // 2))])
        sl = slots.to(DEV)
        rq.resq_append_kv_cache(k, v, sl, *buf, r)
        back = rq.resq_gather_kv_cache(*buf, sl, r, d_head=d)
        outs = torch.full((2, heads, tokens, d + 8), 9.0, dtype=torch.bfloat16, device=DEV)
        rq.resq_gather_kv_cache(*buf, sl, r, k=outs[0, ..., :d].transpose(0, 1), v=outs[1, ..., :d].transpose(0, 1))
        torch.cuda.synchronize()
        live = [t for t in range(tokens) if 0 <= int(slots[t]) < pages * page]
        for x, b, w, y, o in zip((k, v), buf, was, back, outs):
            rows = rq.resq_quantize_kv_cache(x.reshape(-1, d).contiguous(), r)
            vals = rq.resq_dequantize_kv_cache(rows, d, r).view(tokens, heads, d)
            want, val = w.clone(), torch.zeros_like(vals)
            for t in live:
                want[slots[t] // page, :, slots[t] % page, :nb] = rows.view(tokens, heads, nb)[t]
                val[t] = vals[t]
            assert torch.equal(b, want), "the pages differ from the row quantizer's bytes, or other bytes were written"
            assert torch.equal(y, val) and torch.equal(o[..., :d].transpose(0, 1), val) and bool((o[..., d:] == 9).all())


def test_append_and_gather_without_tokens_and_from_broadcast_heads(rq):
    pages = plain.make_pages(gen(1), 4, 3, 16, 64, 8)
    was = pages.clone()
    none = torch.empty(0, 3, 64, dtype=torch.bfloat16, device=DEV)
    rq.resq_append_kv_cache(none, none, ints([]), pages, pages, 8)
    assert rq.resq_gather_kv_cache(pages, pages, ints([]), 8, d_head=64)[0].shape == (0, 3, 64)
    one = torch.randn(5, 1, 64, generator=gen(2)).to(torch.bfloat16).to(DEV)
    v_pages = pages.clone()
    rq.resq_append_kv_cache(one.expand(-1, 3, -1), one.expand(-1, 3, -1), ints([0, 17, 5, 63, 9]), pages, v_pages, 8)
    assert torch.equal(pages[0, 0, 0], pages[0, 2, 0]) and torch.equal(pages, v_pages) and not torch.equal(pages, was)


def quantized_rows(rq, x, r):
    """Rows of x [n, d] by the row quantizer, each group by itself in a row of its own, filled up with a channel that it has."""
    def group(x, high):
        n = x.shape[1]
        full = torch.cat((x, x[:, :1].expand(-1, -n % 8)), 1).contiguous()
        rows = rq.resq_quantize_kv_cache(full, full.shape[1] if high else 0)
        at = rows.shape[1] - 16 + (0 if high else 8)
        return rows[:, :n if high else n // 2], rows[:, at:at + 8]
    (hi, hi_par), (lo, lo_par) = group(x[:, :r], True), group(x[:, r:], False)
    return torch.cat((hi, lo, hi_par, lo_par), 1)


@pytest.mark.parametrize("d,r", [(96, 12), (64, 20), (8, 4), (128, 124), (256, 4), (200, 100)])
@pytest.mark.parametrize("order", ["head", "token"])
def test_append_and_gather_of_halved_pieces(rq, d, r, order):
    # 8-bit groups of an odd multiple of four channels: rows at even addresses
    for tokens, heads, page, pad in ((1, 1, 1, 0), (67, 5, 24, 0), (300, 3, 16, 4)):
        g = gen(tokens + d + r)
        pages = -(-tokens // page) + 2
        k, v = (torch.randn(tokens, heads, d, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
        k[0] = 2.5
        buf = [plain.make_pages(g, pages, heads, page, d, r, order, pad) for _ in range(2)]
        want = [b.clone() for b in buf]
        slots = torch.randperm(pages * page, generator=g)[:tokens]
        slots[tokens // 2] = -1
        rq.resq_append_kv_cache(k, v, slots.to(torch.int32).to(DEV), *buf, r)
        back = rq.resq_gather_kv_cache(*buf, slots.to(torch.int32).to(DEV), r, d_head=d)
        live = slots >= 0
        for x, b, w, y in zip((k, v), buf, want, back):
            rows = quantized_rows(rq, x.reshape(-1, d), r).view(tokens, heads, -1)
            for t in range(tokens):
                if live[t]:
                    w[slots[t] // page, :, slots[t] % page, :rows.shape[2]] = rows[t]
            assert torch.equal(b, w), "the pages differ from the groups' bytes, or other bytes were written"
            exact = plain.decode_rows(rows, d, r) * live[:, None, None]
            # one rounding to fp32, one to bf16
            assert bool(((y.cpu().double() - exact).abs() <= (2.0 ** -8 + 2.0 ** -20) * exact.abs()).all())


@pytest.mark.parametrize("d,r", [(96, 12), (64, 20), (8, 4), (128, 124), (256, 4), (200, 100), (256, 140), (64, 4), (96, 92), (256, 252)])
@pytest.mark.parametrize("page,order,share", [(16, "head", 4), (24, "token", 1), (16, "token", 12), (1, "head", 8)])
def test_attend_of_halved_pieces(rq, d, r, page, order, share):
    check_attend(rq, *attend_case(51, [300, 0, 1, 129], 2 * share, 2, d, r, page, order), r)


def test_gather_of_repeated_slots(rq):
    pages = [plain.make_pages(gen(n), 4, 3, 16, 64, 8) for n in (3, 4)]
    slots = ints([5, 5, 63, -1, 5, 0, 63])
    every = rq.resq_gather_kv_cache(*pages, ints(list(range(64))), 8, d_head=64)
    k = torch.empty(7, 3, 64, dtype=torch.bfloat16, device=DEV)
    for got, of in zip(rq.resq_gather_kv_cache(*pages, slots, 8, k=k), every):
        want = of[slots.clamp(min=0).long()]
        want[3] = 0
        assert torch.equal(got, want)


def test_slots_beyond_2_gib(rq):
    # pages whose byte offsets pass 32 bits: 5 GB apart
    d, r, page, n = 128, 16, 16, 6
    nb, stride = plain.row_bytes(d, r), 1 << 30
    flat = torch.zeros(2, n * stride, dtype=torch.uint8, device=DEV)
    k_pages, v_pages = (f.as_strided((n, 2, page, nb), (stride, page * nb, nb, 1), f.storage_offset()) for f in flat)
    x = torch.randn(n * page, 2, d, generator=gen(1)).to(torch.bfloat16).to(DEV)
    slots = torch.randperm(n * page, generator=gen(2)).to(torch.int32).to(DEV)
    rq.resq_append_kv_cache(x, -x, slots, k_pages, v_pages, r)
    back = rq.resq_gather_kv_cache(k_pages, v_pages, slots, r, d_head=d)
    rows = rq.resq_quantize_kv_cache(x.view(-1, d), r)
    assert torch.equal(back[0].view(-1, d), rq.resq_dequantize_kv_cache(rows, d, r))
    q = torch.randn(1, 4, d, generator=gen(3)).to(torch.bfloat16).to(DEV)
    table = ints([[5, 0, 4, 1, 3, 2]])
    lse = torch.empty(1, 4, device=DEV)
    out = rq.resq_attend_kv_cache(q, k_pages, v_pages, ints([n * page - 3]), table, r, lse=lse)
    near = [p.contiguous() for p in (k_pages, v_pages)]
    lse2 = torch.empty(1, 4, device=DEV)
    assert torch.equal(out, rq.resq_attend_kv_cache(q, *near, ints([n * page - 3]), table, r, lse=lse2)) and torch.equal(lse, lse2)


# ---- attention -----------------------------------------------------------------------------------

def attend_case(seed, lens, hq, hk, d, r, page, order="head", pad=0, extra_pages=2, poison=True):
    """q, pages, lens, table of a batch; what no sequence owns of the pages is poisoned with 0xFF (codes at their ends, scales
    and zero-points NaN)."""
    g = gen(seed)
    held = [-(-max(n, 0) // page) for n in lens]
    total = sum(held) + extra_pages
    ids = torch.randperm(total, generator=g)
    table = torch.full((len(lens), max(held) + 1), -1, dtype=torch.int32)
    pages = [plain.make_pages(g, total, hk, page, d, r, order, pad, device="cpu") for _ in range(2)]
    used = torch.zeros(total, page, dtype=torch.bool)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = ids[at:at + h].to(torch.int32)
        for i in range(h):
            used[ids[at + i], :min(page, lens[b] - i * page)] = True
        at += h
    if poison:
        for p in pages:
            p[~used[:, None, :].expand(-1, hk, -1)] = 255
    q = torch.randn(len(lens), hq, d, generator=g).to(torch.bfloat16)
    dev = [p.to(DEV) if order == "head" else p.transpose(1, 2).contiguous().to(DEV).transpose(1, 2) for p in pages]
    return q.to(DEV), dev[0], dev[1], ints(lens), table.to(DEV)


def check_attend(rq, q, k_pages, v_pages, lens, table, r, scale=None, softcap=0.0, window=0, **kw):
    lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device=DEV)
    want, want_lse, tol, tol_lse = plain.attend(q, k_pages, v_pages, lens.tolist(), table, r, q.shape[-1] ** -0.5 if scale is None else scale,
                                                softcap, window)
    out = rq.resq_attend_kv_cache(q, k_pages, v_pages, lens, table, r, scale=scale, softcap=softcap, window=window, lse=lse, **kw)
    torch.cuda.synchronize()
    got, got_lse = out.cpu().double(), lse.cpu().double()
    off = (got - want).abs()
    bad = ~(off <= tol + 2.0 ** -8 * (want.abs() + tol))
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), float(off[bad].max()))
    empty = want_lse == -math.inf
    assert torch.equal(empty, got_lse == -math.inf) and not got[empty].any()
    off = (got_lse - want_lse)[~empty].abs()
    assert not (~(off <= tol_lse[~empty])).any(), float((off - tol_lse[~empty]).max())
    return out, lse


LENS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 513, 700, 1025]


@pytest.mark.parametrize("page,order", [(16, "head"), (16, "token"), (1, "head"), (7, "head"), (24, "token"), (32, "head"), (48, "head"),
                                        (64, "head"), (256, "token"), (2048, "head")])
def test_attend_lengths_and_pages(rq, page, order):
    check_attend(rq, *attend_case(page, [0] + LENS + [0], 8, 2, 128, 16, page, order), 16)


@pytest.mark.parametrize("hq,hk", [(1, 1), (4, 4), (7, 7), (6, 2), (8, 2), (32, 8), (7, 1), (8, 1), (9, 1), (16, 1), (17, 1), (24, 1), (40, 2), (33, 3)])
def test_attend_head_layouts(rq, hq, hk):
    for n, lens in enumerate(([1], [129, 0, 40], [1500])):
        check_attend(rq, *attend_case(hq + n, lens, hq, hk, 128, 16, 16), 16)


@pytest.mark.parametrize("d,r", [(128, 0), (128, 8), (128, 24), (128, 32), (128, 64), (128, 120), (128, 128), (64, 8), (64, 0), (64, 64),
                                 (64, 32), (256, 32), (256, 0), (256, 256), (256, 128), (256, 200), (8, 0), (8, 8), (16, 8), (40, 16), (72, 8),
                                 (96, 16), (136, 8), (192, 24), (248, 248)])
@pytest.mark.parametrize("share", [3, 12])
def test_attend_widths(rq, d, r, share):
    check_attend(rq, *attend_case(d + r, [37, 0, 300, 1], 2 * share, 2, d, r, 16), r)
    check_attend(rq, *attend_case(d + r + 1, [77], share, 1, d, r, 24, "token", pad=8), r)


@pytest.mark.parametrize("lens", [[5000], [20000, 3], [131072], [4096] * 20, [1] * 300, [100] * 260 + [9000], [0] * 5])
@pytest.mark.parametrize("share", [1, 8])
def test_attend_long_and_many(rq, lens, share):
    hk = 2 if max(lens) < 50000 else 1
    check_attend(rq, *attend_case(len(lens), lens, hk * share, hk, 64, 8, 64), 8)


@pytest.mark.parametrize("window", [1, 2, 16, 31, 100, 128, 1000, 1 << 40])
@pytest.mark.parametrize("softcap", [0.0, 20.0, 0.5])
def test_attend_window_and_cap(rq, window, softcap):
    for page, order in ((16, "head"), (24, "token")):
        check_attend(rq, *attend_case(window % 97, [0] + LENS, 4, 1, 64, 8, page, order), 8, softcap=softcap, window=window)


@pytest.mark.parametrize("batch", [66, 600, 5001, 65535])
def test_attend_many_sequences_without_tokens(rq, batch):
    """Live sequences at both ends and in the middle of a padded batch; the last time they have more units than there are workgroups, so
    that one's run holds the first one's end (its fifth unit), steps over all the others and holds the last one's beginning."""
    for live in ([(0, 1), (batch - 1, 33)], [(0, 40), (1, 3), (batch // 2, 100), (batch // 2 + 1, 1), (batch - 2, 16), (batch - 1, 700)], [(0, 200), (batch - 1, 120000)]):
        lens = torch.zeros(batch, dtype=torch.int32)
        lens[[b for b, _ in live]] = torch.tensor([n for _, n in live], dtype=torch.int32)
        q, k, v, few, table = attend_case(batch, [n for _, n in live], 2, 1, 16, 8, 256)
        at = lens.nonzero().flatten().to(DEV)
        wide, queries = torch.full((batch, table.shape[1]), -1, dtype=torch.int32, device=DEV), torch.ones(batch, 2, 16, dtype=torch.bfloat16, device=DEV)
        wide[at], queries[at] = table, q
        want, want_lse = check_attend(rq, q, k, v, few, table, 8)
        lse = torch.full((batch, 2), 7.0, device=DEV)
        out = rq.resq_attend_kv_cache(queries, k, v, lens.to(DEV), wide, 8, lse=lse)
        assert torch.equal(out[at], want) and torch.equal(lse[at], want_lse)
        out[at], lse[at] = 0, -math.inf
        assert not out.any() and bool((lse == -math.inf).all())


@pytest.mark.parametrize("hq,hk,d,r", [(9, 1, 64, 8), (16, 1, 128, 16), (34, 2, 128, 16), (4, 1, 128, 16), (8, 2, 256, 32), (24, 2, 256, 256), (3, 3, 96, 12),
                                       (12, 1, 128, 20), (6, 3, 128, 64)])
@pytest.mark.parametrize("window,softcap", [(1, 20.0), (100, 0.0), (129, 5.0), (0, 30.0)])
def test_attend_window_and_cap_of_other_heads(rq, hq, hk, d, r, window, softcap):
    for page, order in ((16, "head"), (24, "token")):
        check_attend(rq, *attend_case(window + d + hq, [0, 1, 33, 130, 700], hq, hk, d, r, page, order), r, softcap=softcap, window=window)


@pytest.mark.parametrize("share", [1, 3, 8, 17])
def test_attend_many_heads_and_many_parts(rq, share):
    # 1024 heads and more, whose queries one workgroup each puts together, some from more parts than a thread reads at once
    lens = torch.randint(0, 90, (300,), generator=gen(share)).tolist() + [20000]
    check_attend(rq, *attend_case(share, lens, 4 * share, 4, 64, 8, 16), 8)


@pytest.mark.parametrize("window", [0, 400000])
def test_attend_runs_of_more_tiles_than_page_entries(rq, window):
    # a workgroup's run of more than 4096 tokens of one head: its wavefronts look up pages a second time
    check_attend(rq, *attend_case(3, [410000] * 8, 2, 1, 8, 0, 16), 0, window=window)


def test_attend_scales(rq):
    case = attend_case(5, [300, 1, 40], 8, 2, 128, 16, 16)
    for scale in (1e-6, 0.02, 3.0, 50.0):   # the last: one token holds all the weight
        check_attend(rq, *case, 16, scale=scale)


def test_attend_pages_that_do_not_exist(rq):
    # entries outside [0, num_pages) take no part, also where that leaves a sequence nothing
    for page, order in ((16, "head"), (32, "head"), (24, "token"), (1, "head")):
        q, k, v, lens, table = attend_case(9, [100, 33, 500, 20], 4, 2, 64, 8, page, order)
        table[0, 1] = -1
        table[1, :] = k.shape[0]
        table[2, ::2] = 2147483647
        table[3, 0] = -2147483648
        check_attend(rq, q, k, v, lens, table, 8)


def test_attend_lengths_outside_the_table(rq):
    q, k, v, lens, table = attend_case(11, [64, 64, 64], 4, 2, 64, 8, 16, extra_pages=8)
    table[:, 4] = torch.arange(3, dtype=torch.int32, device=DEV)   # a row names 80 tokens
    k.copy_(plain.make_pages(gen(1), *k.shape[:3], 64, 8))
    v.copy_(plain.make_pages(gen(2), *k.shape[:3], 64, 8))
    check_attend(rq, q, k, v, ints([2147483647, -2147483648, 81]), table, 8)


def test_attend_strides(rq):
    # queries and outputs inside wider rows, out on q, pages with room between rows, heads and pages, a table inside a wider one
    q, k, v, lens, table = attend_case(12, [333, 0, 64, 2], 8, 2, 128, 16, 16)
    want, want_lse = check_attend(rq, q, k, v, lens, table, 16)
    wide = torch.full((4, 11, 131), 3.0, dtype=torch.bfloat16, device=DEV)
    qs = wide[:, 2:10, 1:129]
    qs.copy_(q)
    big = torch.full((4, 9 + table.shape[1]), -7, dtype=torch.int32, device=DEV)
    big[:, 5:5 + table.shape[1]] = table
    spread = []
    for p in (k, v):
        s = torch.full((p.shape[0] + 1, 3, 20, p.shape[3] + 4), 255, dtype=torch.uint8, device=DEV)
        s[:-1, :2, :16, :p.shape[3]] = p
        spread.append(s[:-1, :2, :16])
    lse = torch.empty(4, 8, device=DEV)
    args = (qs, *spread, lens, big[:, 5:5 + table.shape[1]], 16)
    assert torch.equal(rq.resq_attend_kv_cache(*args, lse=lse), want) and torch.equal(lse, want_lse)
    outs = torch.full((8, 4, 130), 5.0, dtype=torch.bfloat16, device=DEV)
    rq.resq_attend_kv_cache(*args, out=outs[..., :128].transpose(0, 1))
    assert torch.equal(outs[..., :128].transpose(0, 1), want) and bool((outs[..., 128:] == 5).all())
    rq.resq_attend_kv_cache(*args, out=qs)
    assert torch.equal(qs, want)
    wide[:, 2:10, 1:129] = 3.0
    assert bool((wide == 3).all())


def test_attend_values_that_are_not_finite(rq):
    # a NaN or an infinity in a token that is seen reaches the heads that see it, and no others
    q, k, v, lens, table = attend_case(13, [50, 50, 50], 4, 2, 64, 8, 16)
    def poke(pages, b, h, t, at, value):
        nb = plain.row_bytes(64, 8)
        row = pages[table[b, t // 16], h, t % 16]
        row[nb - 16 + 4 * at:nb - 12 + 4 * at] = torch.tensor([value], device=DEV).view(torch.uint8)
    poke(k, 0, 0, 7, 1, float("nan"))     # zero-point of the 8-bit group of a key
    poke(v, 1, 1, 49, 3, float("inf"))    # zero-point of the 4-bit group of a value
    out = rq.resq_attend_kv_cache(q, k, v, lens, table, 8).float()
    assert out[0, :2].isnan().all() and out[0, 2:].isfinite().all()
    assert out[1, :2].isfinite().all() and out[1, 2:, :8].isfinite().all() and not out[1, 2:, 8:].isfinite().any()
    assert out[2].isfinite().all()


def test_attend_weights_keep_their_bits(rq):
    """Few tokens of equal scores (queries of zero): the mean of the values, to the roundings of 32-bit arithmetic and 2^-17 of half the
    values' range.  Sums are of codes with their offsets, at most 143 steps of a 4-bit group and 255 of the 8-bit one, and of zero-points:
    some eight roundings of 2^-24 of the largest partial sum, below 2^-20 of the mean of those magnitudes; weights go in as two bf16
    numbers, each the nearest (2^-8), which leave 2^-17 at most, and that meets the middle of the codes, 7.5 (127.5) steps from their ends."""
    for d, r, hq, hk in ((128, 16, 8, 2), (64, 8, 3, 3), (128, 0, 12, 1), (256, 32, 4, 2), (128, 128, 2, 2), (96, 12, 20, 1)):
        lens = [1, 2, 3, 4, 5, 7] * 6
        q, k, v, lens, table = attend_case(d + r, lens, hq, hk, d, r, 16)
        q.zero_()
        got = rq.resq_attend_kv_cache(q, k, v, lens, table, r).cpu().double()
        low = r + (d - r) // 2
        for b, n in enumerate(lens.tolist()):
            rows = v[table[b, 0].item(), :, :n].cpu()
            par = rows[..., low:low + 16].clone(memory_format=torch.contiguous_format).view(torch.float32).double().abs()
            size = torch.cat(((255 * par[..., 0:1] + par[..., 1:2]).expand(-1, -1, r), (271 * par[..., 2:3] + par[..., 3:4]).expand(-1, -1, d - r)), -1)
            want = plain.decode_rows(rows, d, r).mean(1).repeat_interleave(hq // hk, 0)
            half = torch.cat(((127.5 * par[..., 0:1]).expand(-1, -1, r), (7.5 * par[..., 2:3]).expand(-1, -1, d - r)), -1)
            tol = (2.0 ** -20 * size + 2.0 ** -17 * half).mean(1).repeat_interleave(hq // hk, 0)
            off = (got[b] - want).abs()
            assert not (off > tol + 2.0 ** -8 * (want.abs() + tol)).any(), (d, r, n, float(((off - 2.0 ** -8 * want.abs()) / tol).max()))


def test_attend_equal_calls_give_equal_bits(rq):
    case = attend_case(14, [3000, 10, 7777, 0, 128], 16, 4, 128, 16, 32)
    first = check_attend(rq, *case, 16)
    work = rq.resq_attend_kv_cache_workspace(5, 16, 4, 128)
    for fill in (0, 255, 127):
        work.fill_(fill)   # whatever is left in the workspace
        lse = torch.empty(5, 16, device=DEV)
        assert torch.equal(rq.resq_attend_kv_cache(*case, 16, lse=lse, workspace=work), first[0]) and torch.equal(lse, first[1])


def test_attend_calls_of_many_sizes_share_a_workspace(rq):
    # one after another without a wait between them, each with other heads, lengths and cuts than the one before, and again
    cases = [(attend_case(31, [3000, 10, 7777, 0, 128], 16, 4, 128, 16, 32), 16), (attend_case(32, [40000], 8, 1, 64, 8, 16), 8),
             (attend_case(33, [700] * 40, 6, 6, 64, 8, 24, "token"), 8), (attend_case(34, [900, 5, 2000], 34, 2, 96, 0, 16), 0),
             (attend_case(35, [0, 0], 2, 1, 64, 8, 16), 8), (attend_case(36, [1500, 1400], 4, 2, 256, 32, 16), 32)]
    work = max((rq.resq_attend_kv_cache_workspace(*case[0].shape[:2], case[1].shape[1], case[0].shape[2]) for case, _ in cases), key=len)
    want = [check_attend(rq, *case, r)[0] for case, r in cases]
    torch.cuda.synchronize()
    got = [[rq.resq_attend_kv_cache(*case, r, workspace=work) for case, r in cases] for _ in range(30)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for round_ in got for a, b in zip(round_, want))


def test_attend_on_other_streams(rq):
    case = attend_case(15, [3000, 10, 777], 16, 4, 128, 16, 32)
    want = check_attend(rq, *case, 16)[0]
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for n in range(8):   # two calls at once, each with a workspace of its own
        outs.append(torch.empty_like(want))
        rq.resq_attend_kv_cache(*case, 16, out=outs[-1], stream=side[n % 2])
    with torch.cuda.stream(side[0]):
        outs.append(rq.resq_attend_kv_cache(*case, 16))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_buffers_that_a_call_makes_on_another_stream(rq):
    """Outputs and workspace that a call on `stream` makes for itself are not blocks that the current stream has work on: that work
    would land in them behind the call.  The stream as an object, as a handle, and as the default stream's handle, 0."""
    case = attend_case(17, [3000, 10, 777], 16, 4, 128, 16, 32)
    x, freq = torch.randn(300, 6, 128, generator=gen(18)).to(torch.bfloat16).to(DEV), rq.resq_rope_frequencies(128)[0]
    positions, slots = ints(list(range(300))), ints(list(range(0, 96, 2)))
    calls = [lambda s: (rq.resq_attend_kv_cache(*case, 16, stream=s),), lambda s: (rq.resq_rope_heads(x, positions, freq, stream=s),),
             lambda s: rq.resq_gather_kv_cache(case[1], case[2], slots, 16, d_head=128, stream=s)]
    want = [f(None) for f in calls]
    sizes = {t.nbytes for ts in want for t in ts} | {rq.resq_attend_kv_cache_workspace_bytes(3, 16, 4, 128)}
    side, own = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream, current in ((side, own), (side.cuda_stream, own), (0, own), (side, torch.cuda.default_stream())):
        with torch.cuda.stream(current):
            for f, expected in zip(calls, want):
                busy = torch.randn(2048, 2048, device=DEV)
                for _ in range(40):
                    busy = busy @ busy * 1e-2
                junk = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(4)]
                for j in junk:
                    j.fill_(255)   # behind what is running
                del junk, j
                got = f(stream)
                torch.cuda.synchronize()
                assert len(got) == len(expected) and all(torch.equal(a, b) for a, b in zip(got, expected))


def test_calls_without_tokens_on_another_stream(rq):
    side, freq = torch.cuda.Stream(), rq.resq_rope_frequencies(64)[0]
    none = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    pages = [torch.zeros(3, 2, 16, 52, dtype=torch.uint8, device=DEV) for _ in range(2)]
    assert rq.resq_rope_heads(none, ints([]), freq, stream=side).shape == (0, 2, 64)
    assert rq.resq_gather_kv_cache(*pages, ints([]), 8, d_head=64, stream=side)[1].shape == (0, 2, 64)
    assert rq.resq_attend_kv_cache(none, *pages, ints([]), torch.empty(0, 3, dtype=torch.int32, device=DEV), 8, stream=side).shape == (0, 2, 64)


def test_buffers_that_a_captured_call_makes_on_another_stream(rq):
    # a side stream that forks off the capture and comes back to it; replays with the program's own work and allocations between them
    case = attend_case(19, [300, 10, 777], 16, 4, 128, 16, 32)
    x, freq, positions = torch.randn(300, 6, 128, generator=gen(18)).to(torch.bfloat16).to(DEV), rq.resq_rope_frequencies(128)[0], ints(list(range(300)))
    want = rq.resq_attend_kv_cache(*case, 16), rq.resq_rope_heads(x, positions, freq)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        got = rq.resq_attend_kv_cache(*case, 16, stream=side), rq.resq_rope_heads(x, positions, freq, stream=side)
        torch.cuda.current_stream().wait_stream(side)
    for _ in range(4):
        junk = [torch.full_like(t, 5) for t in got for _ in range(4)]
        for t in got:
            t.fill_(7)
        graph.replay()
        again = rq.resq_attend_kv_cache(*case, 16, stream=side), rq.resq_rope_heads(x, positions, freq, stream=side)
        del junk
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got + again, want + want))


def test_attend_graphs_share_a_workspace(rq):
    # two captured calls, one with rows of 16 KB in LDS per wavefront, replayed in turn with eager calls between them
    cases = [(attend_case(41, [900, 0, 33], 4, 2, 256, 256, 16), 256), (attend_case(42, [5000, 77], 16, 2, 128, 16, 24, "token"), 16)]
    work = max((rq.resq_attend_kv_cache_workspace(*case[0].shape[:2], case[1].shape[1], case[0].shape[2]) for case, _ in cases), key=len)
    outs = [torch.empty_like(case[0]) for case, _ in cases]
    graphs = []
    for (case, r), out in zip(cases, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            rq.resq_attend_kv_cache(*case, r, out=out, workspace=work)
    want = [check_attend(rq, *case, r)[0] for case, r in cases]
    for _ in range(4):
        for k in (0, 1, 1, 0):
            outs[k].fill_(7)
            graphs[k].replay()
            rq.resq_attend_kv_cache(*cases[1 - k][0], cases[1 - k][1], workspace=work)
            torch.cuda.synchronize()
            assert torch.equal(outs[k], want[k])


# ---- a step of generation ------------------------------------------------------------------------

def test_steps_of_generation(rq):
    """Prompts, then tokens one by one: plan, norm and rotation, projection onto the cache basis, paged writer, attention, as a
    program runs them; the single-token step captured and replayed.  Each attention against the 64-bit one on the pages, and the
    pages against the row quantizer of what the step before it wrote."""
    batch, hq, hk, d, r, page, steps = 6, 8, 2, 128, 16, 16, 9
    heads, width, total = hq + hk, 8, 40
    g = gen(21)
    free, table, p = torch.randperm(total, generator=g).to(torch.int32).to(DEV), torch.full((batch, width), -1, dtype=torch.int32, device=DEV), None
    pages = [torch.full((total, hk, page, plain.row_bytes(d, r)), 255, dtype=torch.uint8, device=DEV) for _ in range(2)]
    freq, mscale = rq.resq_rope_frequencies(d, base=500000.0, scaling="bands", factor=8.0)
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(torch.bfloat16).to(DEV) for _ in range(2)]
    basis = rq.resq_pack_weights(torch.linalg.qr(torch.randn(d, d, generator=g))[0].contiguous().to(torch.bfloat16).to(DEV), d)
    keys, values = {}, {}   # slot -> row bytes

    def step(qkv, plan, y):
        rq.resq_rope_heads(qkv[:, :heads], plan.positions, freq, heads_q=hq, w_q=w[0], w_k=w[1], mscale=mscale, out=y)
        z = rq.resq_project_heads(y.view(-1, d), basis).view(y.shape)
        rq.resq_append_kv_cache(z[:, hq:], qkv[:, heads:], plan.slots, *pages, r)
        return z

    def record(plan, z, qkv):
        for x, rows in ((z[:, hq:], keys), (qkv[:, heads:], values)):
            got = rq.resq_quantize_kv_cache(x.reshape(-1, d).contiguous(), r).view(len(x), hk, -1)
            for t, s in enumerate(plan.slots.tolist()):
                if s >= 0:
                    rows[s] = got[t]

    def pages_hold(rows, pages):
        want = torch.full_like(pages, 255)
        for s, x in rows.items():
            want[s // page, :, s % page] = x
        return torch.equal(pages, want)

    # prompts of ragged lengths, one of them empty so far, in one padded batch
    news = ints([20, 1, 0, 33, 16, 7])
    first = rq.KvSlots(batch, 90)
    rq.resq_kv_slots(first.lens, news, free, None, table, page, total, out=first)
    assert first.state.tolist()[1] == 0
    qkv = torch.randn(90, heads + hk, d, generator=g).to(torch.bfloat16).to(DEV)
    record(first, step(qkv, first, torch.empty(90, heads, d, dtype=torch.bfloat16, device=DEV)), qkv)
    assert pages_hold(keys, pages[0]) and pages_hold(values, pages[1])

    # then a token each: a captured step that goes on from its own lengths
    p = rq.KvSlots(batch, batch)
    p.lens.copy_(first.lens)
    p.state.copy_(first.state)
    ones, qkv = ints([1] * batch), torch.empty(batch, heads + hk, d, dtype=torch.bfloat16, device=DEV)
    y, out, lse = torch.empty(batch, heads, d, dtype=torch.bfloat16, device=DEV), torch.empty(batch, hq, d, dtype=torch.bfloat16, device=DEV), \
        torch.empty(batch, hq, device=DEV)
    work = rq.resq_attend_kv_cache_workspace(batch, hq, hk, d)

    def token():
        rq.resq_kv_slots(p.lens, ones, free, None, table, page, total, out=p)
        z = step(qkv, p, y)
        rq.resq_attend_kv_cache(z[:, :hq], *pages, p.lens, table, r, out=out, lse=lse, workspace=work)
        return z

    kept = {k: v.clone() for k, v in (("lens", p.lens), ("state", p.state), ("table", table))}
    qkv.copy_(torch.randn(qkv.shape, generator=g))
    token()                                                   # eager once, and back: a captured step must find everything loaded
    p.lens.copy_(kept["lens"])
    p.state.copy_(kept["state"])
    table.copy_(kept["table"])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z = token()
    for n in range(steps):
        qkv.copy_(torch.randn(qkv.shape, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        assert p.state.tolist()[1] == 0 and p.lens.tolist() == [a + n + 1 for a in (20, 1, 0, 33, 16, 7)]
        record(p, z, qkv)
        assert pages_hold(keys, pages[0]) and pages_hold(values, pages[1])
        replayed, replayed_lse = out.clone(), lse.clone()
        eager, eager_lse = check_attend(rq, z[:, :hq], *pages, p.lens, table, r)
        assert torch.equal(eager, replayed) and torch.equal(eager_lse, replayed_lse)
