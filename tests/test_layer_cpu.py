"""What the entry points around a layer's products refuse, and their host functions, without a GPU."""
import pytest
import torch

from paper_2412_14363_amd import binding

P = 0x10000   # a plausible, aligned, never dereferenced address
OK, NULL, SHAPE, ALIGN, BUFFER = 0, 1, 2, 3, 4


def call(name, good, **change):
    """The entry point with the arguments of `good` (in order), some changed."""
    assert set(change) <= set(good)
    return getattr(binding.lib(), name)(*{**good, **change}.values())


PROMPTS = dict(q=P, ldq=1024, ldqh=128, tokens_q=40, k=P, ldk=256, ldkh=128, v=P, ldv=256, ldvh=128, tokens_k=50, cu_q=P, cu_k=P, B=3, heads_q=8,
               heads_k=2, d=128, scale=0.1, softcap=0.0, window=0, out=P, ldo=1024, ldoh=128, lse=None, workspace=P, nbytes=1 << 40, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens_q=-1), SHAPE), (dict(tokens_k=-1), SHAPE), (dict(tokens_q=(1 << 30) + 1, heads_q=1, heads_k=1), SHAPE), (dict(tokens_k=(1 << 30) + 1), SHAPE),
    (dict(tokens_q=1 << 30), SHAPE), (dict(B=0), SHAPE), (dict(B=65536), SHAPE), (dict(heads_q=7), SHAPE), (dict(heads_k=0), SHAPE),
    (dict(heads_q=0), SHAPE), (dict(heads_q=70000, heads_k=70000), SHAPE), (dict(d=4), SHAPE), (dict(d=100), SHAPE), (dict(d=264), SHAPE),
    (dict(ldq=-1), SHAPE), (dict(ldkh=-8), SHAPE), (dict(ldv=-8), SHAPE), (dict(ldk=1 << 24), SHAPE), (dict(ldv=1 << 40), SHAPE), (dict(ldoh=100), SHAPE), (dict(ldo=1023), SHAPE), (dict(scale=0.0), SHAPE),
    (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(softcap=-1.0), SHAPE),
    (dict(softcap=float("nan")), SHAPE), (dict(softcap=1e-39), SHAPE), (dict(window=-1), SHAPE), (dict(ldq=2048), SHAPE),
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(v=None), NULL), (dict(cu_q=None), NULL), (dict(cu_k=None), NULL), (dict(out=None), NULL),
    (dict(workspace=None), NULL), (dict(q=P + 1), ALIGN), (dict(out=2 * P + 1), ALIGN), (dict(k=P + 8), ALIGN), (dict(v=P + 2), ALIGN),
    (dict(ldk=260), ALIGN), (dict(ldvh=132), ALIGN), (dict(cu_q=P + 2), ALIGN), (dict(cu_k=P + 1), ALIGN), (dict(lse=P + 2), ALIGN),
    (dict(workspace=P + 16), ALIGN), (dict(nbytes=8), BUFFER), (dict(tokens_q=0, q=None, out=None, workspace=None), OK)])
def test_prompts_refuses(change, status):
    assert call("resq_attend_prompts", PROMPTS, **change) == status


def test_prompts_workspace_sizes():
    f = binding.resq_attend_prompts_workspace_bytes
    assert f(1, 1, 1, 32, 8, 128) > 0 and f(300, 100000, 1, 32, 8, 128) > f(300, 300, 1, 32, 8, 128) and f(0, 0, 65535, 8, 8, 256) > 0
    for bad in ((-1, 1, 1, 8, 8, 64), (1, -1, 1, 8, 8, 64), (1, 1, 0, 8, 8, 64), (1, 1, 65536, 8, 8, 64), (1, 1, 1, 8, 3, 64), (1, 1, 1, 8, 0, 64),
                (1, 1, 1, 8, 8, 60), (1, 1, 1, 8, 8, 264), (1 << 30, 1, 1, 8, 8, 64)):
        assert f(*bad) == 0, bad
    with pytest.raises(ValueError):
        binding.resq_attend_prompts_workspace(1, 1, 1, 8, 3, 64)


def test_prompts_binding_refuses():
    bf16, i32 = torch.bfloat16, torch.int32
    q, k, cu = torch.zeros(4, 8, 64, dtype=bf16), torch.zeros(5, 2, 64, dtype=bf16), torch.zeros(3, dtype=i32)
    space = torch.zeros(256, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device memory"):   # everything fits but where it lives
        binding.resq_attend_prompts(q, k, k, cu, workspace=space)
    for args, kw in (((q.float(), k, k, cu), {}), ((q.transpose(1, 2), k, k, cu), {}), ((q, k, k[:4], cu), {}), ((q, k[:, :, :32], k[:, :, :32], cu), {}),
                     ((q, k.repeat(1, 2, 1)[:, :3], k.repeat(1, 2, 1)[:, :3], cu), {}), ((q, k, k, cu.long()), {}), ((q, k, k, cu, cu[:2]), {}),
                     ((q, k, k, cu[:1]), {}), ((q, k, k, cu), dict(out=q[:3])), ((q, k, k, cu), dict(lse=torch.zeros(4, 2))),
                     ((q, k[0], k[0], cu), {})):
        with pytest.raises(ValueError):
            binding.resq_attend_prompts(*args, workspace=space, **kw)


NORM = dict(y=P, ldy=512, gate=P, ldg=0, h=2 * P, ldh=512, h_is_fp32=0, tokens=4, width=512, w_pre=P, w_post=P, w_offset=0.0, eps=1e-6, alpha=1.0,
            h_out=3 * P, ldho=512, x=4 * P, ldx=512, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(tokens=-1), SHAPE), (dict(width=0), SHAPE), (dict(width=32769, ldho=40000, ldx=40000), SHAPE), (dict(ldy=-1), SHAPE), (dict(ldg=-1), SHAPE),
    (dict(ldh=-1), SHAPE), (dict(ldho=511), SHAPE), (dict(ldx=100), SHAPE), (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE),
    (dict(eps=float("inf")), SHAPE), (dict(alpha=float("nan")), SHAPE), (dict(w_offset=float("inf")), SHAPE), (dict(h_out=2 * P, ldho=520), SHAPE),
    (dict(x=P, ldx=520), SHAPE), (dict(tokens=1 << 32), SHAPE), (dict(h=None), NULL), (dict(h_out=None, x=None), NULL), (dict(w_pre=None), NULL),
    (dict(y=None), NULL), (dict(y=None, gate=None), NULL), (dict(y=P + 1), ALIGN), (dict(gate=P + 1), ALIGN), (dict(h=2 * P + 1), ALIGN),
    (dict(h=2 * P + 2, h_is_fp32=1), ALIGN), (dict(h_out=3 * P + 2, h_is_fp32=1), ALIGN), (dict(x=4 * P + 1), ALIGN), (dict(w_pre=P + 1), ALIGN),
    (dict(w_post=P + 1), ALIGN), (dict(tokens=0, h=None), OK)])
def test_norm_refuses(change, status):
    assert call("resq_norm_residual", NORM, **change) == status


def test_norm_binding_refuses():
    bf16 = torch.bfloat16
    y, w = torch.zeros(4, 64, dtype=bf16), torch.zeros(64, dtype=bf16)
    with pytest.raises(ValueError, match="device memory"):
        binding.resq_norm_residual(y, y, w)
    for args, kw in (((y, y.half(), w), {}), ((y.float(), y, w), {}), ((y[:3], y, w), {}), ((y, y, w[:32]), {}), ((y, y, w.float()), {}),
                     ((y, y, w), dict(w_post=w[:32])), ((y, y, w), dict(gate=y[:2])), ((None, y, w), dict(gate=w)), ((None, y, w), dict(w_post=w)),
                     ((y, y, None), dict(x=y)), ((y, y, w), dict(h_out=y.float())), ((y, y, w), dict(x=y[:2])), ((y, y.t().contiguous().t(), w), {})):
        with pytest.raises(ValueError):
            binding.resq_norm_residual(*args, **kw)


PREFIX = dict(q=P, ldq=4096, ldqh=128, B=4, heads_q=32, heads_k=8, d=128, r=16, prefix_len=P, prefix_table=P, prefix_width=7, lens=P, table=P,
              ld_table=10, width=10, k_pages=P, v_pages=P, num_pages=10, page_size=16, page_stride=8 * 16 * 88, head_stride=16 * 88, row_stride=88,
              scale=0.1, softcap=0.0, window=0, out=P, ldo=4096, ldoh=128, lse=None, workspace=P, nbytes=1 << 40, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(d=124), SHAPE), (dict(d=264), SHAPE), (dict(d=4), SHAPE), (dict(r=136), SHAPE), (dict(r=10), SHAPE), (dict(r=-8), SHAPE), (dict(r=-4), SHAPE),
    (dict(r=12, row_stride=84), BUFFER), (dict(r=12, k_pages=P + 1), ALIGN), (dict(num_pages=0), SHAPE), (dict(page_size=0), SHAPE),
    (dict(num_pages=1 << 27), SHAPE), (dict(row_stride=84), BUFFER), (dict(head_stride=80), BUFFER), (dict(page_stride=0), BUFFER),
    (dict(k_pages=None), NULL), (dict(v_pages=None), NULL), (dict(k_pages=P + 2), ALIGN), (dict(row_stride=90), ALIGN), (dict(B=0), SHAPE),
    (dict(B=70000), SHAPE), (dict(heads_q=31), SHAPE), (dict(heads_k=0), SHAPE), (dict(ldq=-1), SHAPE), (dict(ldoh=64), SHAPE), (dict(ldo=4095), SHAPE),
    (dict(prefix_width=0), SHAPE), (dict(prefix_width=1 << 31), SHAPE), (dict(width=0), SHAPE), (dict(width=11), SHAPE), (dict(scale=0.0), SHAPE),
    (dict(scale=float("nan")), SHAPE), (dict(softcap=-1.0), SHAPE), (dict(softcap=1e-39), SHAPE), (dict(window=-1), SHAPE), (dict(ldq=8192), SHAPE),
    (dict(q=None), NULL), (dict(prefix_len=None), NULL), (dict(prefix_table=None), NULL), (dict(lens=None), NULL), (dict(table=None), NULL),
    (dict(out=None), NULL), (dict(workspace=None), NULL), (dict(q=P + 1), ALIGN), (dict(out=2 * P + 1), ALIGN), (dict(prefix_len=P + 2), ALIGN),
    (dict(prefix_table=P + 1), ALIGN), (dict(lens=P + 2), ALIGN), (dict(table=P + 2), ALIGN), (dict(lse=P + 2), ALIGN), (dict(workspace=P + 16), ALIGN),
    (dict(nbytes=64), BUFFER), (dict(B=65535, heads_q=512, heads_k=512, ldo=65536, ldq=65536), SHAPE)])
def test_prefix_refuses(change, status):
    assert call("resq_attend_kv_prefix", PREFIX, **change) == status


def test_prefix_workspace_sizes():
    f, own = binding.resq_attend_kv_prefix_workspace_bytes, binding.resq_attend_kv_cache_workspace_bytes
    assert f(1, 32, 8, 128) > own(1, 32, 8, 128) and f(64, 32, 8, 128) > own(64, 32, 8, 128)
    assert f(0, 32, 8, 128) == f(1, 31, 8, 128) == f(1, 32, 8, 264) == f(1, 32, 8, 100) == f(65536, 8, 8, 64) == f(1, 8, 0, 64) == 0
    with pytest.raises(ValueError):
        binding.resq_attend_kv_prefix_workspace(1, 31, 8, 128)


def test_prefix_binding_refuses():
    i32, bf16 = torch.int32, torch.bfloat16
    q, n, pages, table = torch.zeros(4, 2, 64, dtype=bf16), torch.zeros(4, dtype=i32), torch.zeros(3, 2, 16, 52, dtype=torch.uint8), torch.zeros(4, 3, dtype=i32)
    space = torch.zeros(256, dtype=torch.uint8)
    f = binding.resq_attend_kv_prefix
    with pytest.raises(ValueError, match="device memory"):
        f(q, pages, pages, n[:1], n, n, table, 8, workspace=space)
    for args, kw in (((q.float(), pages, pages, n[:1], n, n, table, 8), {}), ((q[:, :1], pages, pages, n[:1], n, n, table, 8), {}),
                     ((q, pages, pages[:2], n[:1], n, n, table, 8), {}), ((q, pages, pages, n[:2], n, n, table, 8), {}),
                     ((q, pages, pages, n[:1], table, n, table, 8), {}), ((q, pages, pages, n[:1], n.long(), n, table, 8), {}),
                     ((q, pages, pages, n[:1], n, n[:3], table, 8), {}), ((q, pages, pages, n[:1], n, n, table[:3], 8), {}),
                     ((q, pages, pages, n[:1], n, n, table, 64), {}), ((q, pages, pages, n[:1], n[:0], n, table, 8), {}),
                     ((q, pages, pages, n[:1], n, n, table, 8), dict(lse=torch.zeros(4, 3))), ((q, pages, pages, n[:1], n, n, table, 8), dict(out=q[:2]))):
        with pytest.raises(ValueError):
            f(*args, workspace=space, **kw)
