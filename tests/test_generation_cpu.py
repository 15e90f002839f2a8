"""What the generation step's entry points refuse, and their host functions, without a GPU."""
import ctypes as C
import math

import pytest
import torch

from paper_2412_14363_amd import binding

P = 0x10000   # a plausible, aligned, never dereferenced address
OK, NULL, SHAPE, ALIGN, BUFFER = 0, 1, 2, 3, 4


def call(name, good, **change):
    """The entry point with the arguments of `good` (in order), some changed."""
    assert set(change) <= set(good)
    return getattr(binding.lib(), name)(*{**good, **change}.values())


SLOTS = dict(lens=P, news=P, B=4, page_size=16, num_pages=100, free=P, n_free=50, taken=P, table=P, ld_table=10, width=10, max_tokens=64,
             lens_out=P, cu_tokens=P, cu_pages=P, positions=P, slots=P, state=P, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(B=0), SHAPE), (dict(B=65537), SHAPE), (dict(page_size=0), SHAPE), (dict(num_pages=0), SHAPE), (dict(num_pages=1 << 27), SHAPE),
    (dict(n_free=-1), SHAPE), (dict(width=0), SHAPE), (dict(width=11), SHAPE), (dict(width=1 << 27, ld_table=1 << 27), SHAPE),
    (dict(max_tokens=0), SHAPE), (dict(max_tokens=(1 << 31) - 1), SHAPE), (dict(lens=None), NULL), (dict(news=None), NULL),
    (dict(free=None), NULL), (dict(taken=None), NULL), (dict(table=None), NULL), (dict(lens_out=None), NULL), (dict(cu_tokens=None), NULL),
    (dict(cu_pages=None), NULL), (dict(positions=None), NULL), (dict(slots=None), NULL), (dict(state=None), NULL),
    (dict(lens=P + 2), ALIGN), (dict(slots=P + 1), ALIGN), (dict(free=P + 2), ALIGN)])
def test_slots_refuses(change, status):
    assert call("resq_kv_slots", SLOTS, **change) == status


ROPE = dict(x=P, ldx=1280, ldxh=128, tokens=8, heads_q=8, heads_k=2, d=128, w_q=P, w_k=P, eps=1e-6, positions=P, freq=P, rot=128,
            interleaved=0, mscale=1.0, y=P, ldy=1280, ldyh=128, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), SHAPE), (dict(heads_q=0, heads_k=0), SHAPE), (dict(heads_q=-1), SHAPE), (dict(heads_k=70000), SHAPE), (dict(d=127), SHAPE),
    (dict(d=514, ldxh=514, ldyh=514, ldx=5140, ldy=5140), SHAPE), (dict(rot=130), SHAPE), (dict(rot=127), SHAPE), (dict(rot=-2), SHAPE),
    (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE), (dict(ldx=-1), SHAPE), (dict(ldyh=120), SHAPE),
    (dict(ldy=1279), SHAPE), (dict(ldy=128, ldyh=1000, y=2 * P), SHAPE), (dict(ldx=1288), SHAPE), (dict(x=None), NULL),
    (dict(y=None), NULL), (dict(positions=None), NULL), (dict(freq=None), NULL), (dict(w_q=None), NULL), (dict(w_k=None), NULL),
    (dict(x=P + 1), ALIGN), (dict(freq=P + 4), ALIGN), (dict(w_q=P + 1), ALIGN), (dict(positions=P + 2), ALIGN), (dict(tokens=0, x=None), OK),
    (dict(tokens=1 << 29, heads_q=1, heads_k=0), SHAPE), (dict(tokens=1 << 30, x=P + 2), SHAPE)])   # more threads than a launch counts
def test_rope_refuses(change, status):
    assert call("resq_rope_heads", ROPE, **change) == status


APPEND = dict(k=P, ldk=1024, ldkh=128, v=P, ldv=1024, ldvh=128, tokens=4, heads=8, d=128, r=16, slots=P, k_pages=P, v_pages=P, num_pages=10,
              page_size=16, page_stride=8 * 16 * 88, head_stride=16 * 88, row_stride=88, stream=None)
PAGE_FAULTS = [
    (dict(d=124), SHAPE), (dict(d=520), SHAPE), (dict(r=136), SHAPE), (dict(r=10), SHAPE), (dict(r=-8), SHAPE),
    (dict(r=-4), SHAPE),
    (dict(r=12, row_stride=91, head_stride=1456, page_stride=11648), ALIGN), (dict(r=12, row_stride=84), BUFFER),
    (dict(r=12, k_pages=P + 1), ALIGN), (dict(num_pages=0), SHAPE),
    (dict(page_size=0), SHAPE), (dict(num_pages=1 << 27), SHAPE), (dict(row_stride=84), BUFFER),
    (dict(head_stride=80), BUFFER), (dict(page_stride=0), BUFFER), (dict(k_pages=None), NULL), (dict(v_pages=None), NULL),
    (dict(k_pages=P + 2), ALIGN), (dict(v_pages=P + 1), ALIGN), (dict(row_stride=90), ALIGN), (dict(head_stride=1410), ALIGN),
    (dict(page_stride=12345 * 2), ALIGN)]


@pytest.mark.parametrize("change,status", PAGE_FAULTS + [
    (dict(tokens=-1), SHAPE), (dict(heads=0), SHAPE), (dict(ldk=-8), SHAPE), (dict(k=None), NULL), (dict(v=None), NULL), (dict(slots=None), NULL),
    (dict(k=P + 8), ALIGN), (dict(v=P + 2), ALIGN), (dict(ldk=1028), ALIGN), (dict(ldv=2048, ldvh=132), ALIGN), (dict(slots=P + 2), ALIGN),
    (dict(tokens=0, k=None, slots=None), OK), (dict(tokens=1 << 28), SHAPE),
    (dict(d=264, r=12, ldk=2112, ldkh=264, ldv=2112, ldvh=264, row_stride=512, head_stride=8192, page_stride=1 << 17), SHAPE), (dict(tokens=1 << 25), SHAPE),
    (dict(tokens=1 << 24, d=256, ldk=2048, ldkh=256, ldv=2048, ldvh=256, row_stride=256, head_stride=4096, page_stride=32768), SHAPE)])
def test_append_and_gather_refuse(change, status):
    assert call("resq_append_kv_cache", APPEND, **change) == status
    order = ["k_pages", "v_pages", "num_pages", "page_size", "page_stride", "head_stride", "row_stride", "slots", "tokens", "heads", "d", "r",
             "k", "ldk", "ldkh", "v", "ldv", "ldvh", "stream"]
    assert call("resq_gather_kv_cache", {n: APPEND[n] for n in order}, **change) == status


def test_gather_refuses_rows_that_overlap():
    order = ["k_pages", "v_pages", "num_pages", "page_size", "page_stride", "head_stride", "row_stride", "slots", "tokens", "heads", "d", "r",
             "k", "ldk", "ldkh", "v", "ldv", "ldvh", "stream"]
    good = {n: APPEND[n] for n in order}
    for change in (dict(ldk=0), dict(ldvh=0), dict(ldk=512), dict(ldv=128, ldvh=256)):
        assert call("resq_gather_kv_cache", good, **change) == SHAPE


ATTEND = dict(q=P, ldq=4096, ldqh=128, B=4, heads_q=32, heads_k=8, d=128, r=16, lens=P, table=P, ld_table=10, width=10, k_pages=P, v_pages=P,
              num_pages=10, page_size=16, page_stride=8 * 16 * 88, head_stride=16 * 88, row_stride=88, scale=0.1, softcap=0.0, window=0, out=P,
              ldo=4096, ldoh=128, lse=None, workspace=P, nbytes=1 << 40, stream=None)


@pytest.mark.parametrize("change,status", PAGE_FAULTS + [
    (dict(B=0), SHAPE), (dict(B=70000), SHAPE), (dict(heads_q=31), SHAPE), (dict(heads_k=0), SHAPE), (dict(d=264), SHAPE), (dict(d=4), SHAPE),
    (dict(ldq=-1), SHAPE), (dict(ldoh=64), SHAPE), (dict(ldo=4095), SHAPE), (dict(width=0), SHAPE), (dict(width=11), SHAPE),
    (dict(scale=0.0), SHAPE), (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE),
    (dict(softcap=-1.0), SHAPE), (dict(softcap=float("nan")), SHAPE), (dict(window=-1), SHAPE), (dict(q=None), NULL), (dict(lens=None), NULL),
    (dict(table=None), NULL), (dict(out=None), NULL), (dict(workspace=None), NULL), (dict(q=P + 1), ALIGN), (dict(out=P + 1), ALIGN),
    (dict(lens=P + 2), ALIGN), (dict(table=P + 2), ALIGN), (dict(lse=P + 2), ALIGN), (dict(workspace=P + 16), ALIGN), (dict(nbytes=64), BUFFER),
    (dict(B=65535, heads_q=512, heads_k=512, ldo=65536), SHAPE), (dict(softcap=1e-39), SHAPE)])
def test_attend_refuses(change, status):
    assert call("resq_attend_kv_cache", ATTEND, **change) == status


def test_attend_workspace_sizes():
    f = binding.resq_attend_kv_cache_workspace_bytes
    assert f(1, 32, 8, 128) > 0 and f(64, 32, 8, 128) >= f(1, 32, 8, 128) and f(65535, 8, 8, 256) > 0
    assert f(0, 32, 8, 128) == f(1, 31, 8, 128) == f(1, 32, 8, 264) == f(1, 32, 8, 100) == f(65536, 8, 8, 64) == f(1, 8, 0, 64) == 0


def test_binding_refuses_host_tensors_and_wrong_types():
    i32, bf16 = torch.int32, torch.bfloat16
    x, slots, pages = torch.zeros(4, 2, 64, dtype=bf16), torch.zeros(4, dtype=i32), torch.zeros(3, 2, 16, 52, dtype=torch.uint8)
    table, freq = torch.zeros(4, 3, dtype=i32), torch.zeros(32, dtype=torch.float64)
    calls = [lambda: binding.resq_rope_heads(x, slots, freq), lambda: binding.resq_append_kv_cache(x, x, slots, pages, pages, 8),
             lambda: binding.resq_gather_kv_cache(pages, pages, slots, 8, d_head=64),
             lambda: binding.resq_attend_kv_cache(x, pages, pages, slots, table, 8),
             lambda: binding.resq_kv_slots(slots, slots, slots, slots[:1], table, 16, 3, out=binding.KvSlots(4, 8, device="cpu"))]
    for f in calls:   # everything fits but where it lives
        with pytest.raises(ValueError, match="device memory"):
            f()
    for f in (lambda: binding.resq_rope_heads(x.float(), slots, freq), lambda: binding.resq_rope_heads(x.transpose(1, 2), slots, freq),
              lambda: binding.resq_append_kv_cache(x, x[:3], slots, pages, pages, 8),
              lambda: binding.resq_gather_kv_cache(pages, pages, slots, 8), lambda: binding.resq_gather_kv_cache(pages[0], pages[0], slots, 8, d_head=64),
              lambda: binding.resq_gather_kv_cache(pages, pages, slots, 8, k=x[:3], v=x[:3]),
              lambda: binding.resq_attend_kv_cache(x[:, :1], pages, pages, slots, table, 8),
              lambda: binding.resq_attend_kv_cache(x, pages, pages, slots, table, 8, lse=torch.zeros(4, 2, dtype=torch.float64)),
              lambda: binding.resq_kv_slots(slots, slots, slots, slots[:1], table, 16, 3)):
        with pytest.raises(ValueError):
            f()


def frequencies(rot, **kw):
    f, m = binding.resq_rope_frequencies(rot, device="cpu", **kw)
    return f.tolist(), m


def test_rope_frequencies():
    plain, m = frequencies(128, base=500000.0)
    assert m == 1.0 and all(math.isclose(f, 500000.0 ** (-i / 64), rel_tol=1e-14) for i, f in enumerate(plain))
    linear, m = frequencies(128, base=500000.0, scaling="linear", factor=4.0)
    assert m == 1.0 and all(math.isclose(4 * a, b, rel_tol=1e-14) for a, b in zip(linear, plain))
    base, m = frequencies(128, base=500000.0, scaling="base", factor=4.0)   # ends: the fastest stays, the slowest is a quarter
    assert m == 1.0 and base[0] == plain[0] and math.isclose(4 * base[-1], plain[-1], rel_tol=1e-12)
    bands, m = frequencies(128, base=500000.0, scaling="bands", factor=8.0, low=1.0, high=4.0, original_len=8192)
    assert m == 1.0
    for a, b in zip(bands, plain):
        turns = 8192 * b / (2 * math.pi)
        if turns >= 4:
            assert a == b
        elif turns <= 1:
            assert math.isclose(8 * a, b, rel_tol=1e-14)
        else:
            s = (turns - 1) / 3
            assert math.isclose(a, s * b + (1 - s) * b / 8, rel_tol=1e-12)
    ramp, m = frequencies(64, base=10000.0, scaling="ramp", factor=16.0, low=1.0, high=32.0, original_len=4096)
    assert math.isclose(m, 0.1 * math.log(16) + 1, rel_tol=1e-6)
    pair = lambda turns: 64 * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000.0))
    lo, hi = math.floor(pair(32.0)), math.ceil(pair(1.0))
    for i, a in enumerate(ramp):
        b = 10000.0 ** (-i / 32)
        s = min(max((i - lo) / (hi - lo), 0.0), 1.0)
        assert math.isclose(a, (1 - s) * b + s * b / 16, rel_tol=1e-12)
    assert frequencies(2)[0] == [1.0]


def test_rope_frequencies_refuses():
    f, m, buf = binding.lib().resq_rope_frequencies, C.c_float(), (C.c_double * 256)()
    good = dict(rot=64, base=10000.0, scaling=3, factor=2.0, low=1.0, high=4.0, original_len=4096)
    ask = lambda **kw: f(*{**good, **kw}.values(), buf, C.byref(m))
    assert ask() == OK
    for change in (dict(rot=0), dict(rot=3), dict(rot=514), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(scaling=5),
                   dict(scaling=-1), dict(factor=0.5), dict(factor=float("nan")), dict(low=0.0), dict(high=1.0), dict(original_len=0)):
        assert ask(**change) == SHAPE, change
    assert f(*good.values(), None, C.byref(m)) == NULL and f(*good.values(), buf, None) == NULL
    with pytest.raises(ValueError, match="scaling"):
        binding.resq_rope_frequencies(64, scaling="other", device="cpu")
    with pytest.raises(binding.ResqError, match="RESQ_ERR_SHAPE"):
        binding.resq_rope_frequencies(0, device="cpu")
