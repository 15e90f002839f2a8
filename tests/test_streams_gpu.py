"""Buffers that the layers' and the basis construction's entry points make for themselves on another stream than the current one."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(scope="module")
def rq():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU; there is no CPU fallback")
    from paper_2412_14363_amd import binding
    binding.lib()
    return binding


def tensors(x):
    """What a call has written."""
    if isinstance(x, (torch.Tensor, tuple)):
        return [x] if isinstance(x, torch.Tensor) else list(x)
    return [x.q_hi, x.q_lo, x.s_hi, x.s_lo, x.lo_sum] + ([x.c_hi, x.c_lo] if x.asym else [])


CALLS = ["quantize_act", "hadamard_quantize_act", "quantize_act_asym", "hadamard_quantize_act_asym", "quantize_gemm_mixed", "gemm_mixed",
         "gemm_mixed_asym", "gemm_mixed_swiglu", "pack_weights", "unpack_weights", "gram_accumulate", "sym_eig", "project_rows",
         "project_heads", "quantize_kv_cache", "dequantize_kv_cache", "online_hadamard"]


@pytest.mark.parametrize("name", CALLS)
def test_buffers_that_a_call_makes_on_another_stream(rq, name):
    """They are not blocks that the current stream has work on: that work would land in them behind the call."""
    g = torch.Generator().manual_seed(3)
    bf16 = lambda *shape: torch.randn(*shape, generator=g).to(torch.bfloat16).to(DEV)
    x, w, heads = bf16(9, 1024), bf16(512, 1024), bf16(40, 128)
    packed, square = rq.resq_pack_weights(w, 128), bf16(128, 128)
    basis = rq.resq_pack_weights(square, 128)
    sym, asym, rows = rq.resq_quantize_act(x, 128), rq.resq_quantize_act_asym(x, 128), rq.resq_quantize_kv_cache(heads, 16)
    gram, u = rq.resq_gram_accumulate(heads), torch.randn(1024, 128, generator=g).to(DEV)
    call = {
        "quantize_act": lambda s: rq.resq_quantize_act(x, 128, stream=s),
        "hadamard_quantize_act": lambda s: rq.resq_hadamard_quantize_act(x, 128, stream=s),
        "quantize_act_asym": lambda s: rq.resq_quantize_act_asym(x, 128, stream=s),
        "hadamard_quantize_act_asym": lambda s: rq.resq_hadamard_quantize_act_asym(x, 128, stream=s),
        "quantize_gemm_mixed": lambda s: rq.resq_quantize_gemm_mixed(x, packed, 512, 128, stream=s),
        "gemm_mixed": lambda s: rq.resq_gemm_mixed(sym, packed, 512, stream=s),
        "gemm_mixed_asym": lambda s: rq.resq_gemm_mixed_asym(asym, packed, 512, stream=s),
        "gemm_mixed_swiglu": lambda s: rq.resq_gemm_mixed_swiglu(sym, packed, 512, stream=s),
        "pack_weights": lambda s: rq.resq_pack_weights(w, 128, stream=s),
        "unpack_weights": lambda s: rq.resq_unpack_weights(packed, 512, 1024, 128, stream=s),
        "gram_accumulate": lambda s: rq.resq_gram_accumulate(heads, stream=s),
        "sym_eig": lambda s: rq.resq_sym_eig(gram, stream=s),
        "project_rows": lambda s: rq.resq_project_rows(x, u, stream=s),
        "project_heads": lambda s: rq.resq_project_heads(heads, basis, stream=s),
        "quantize_kv_cache": lambda s: rq.resq_quantize_kv_cache(heads, 16, stream=s),
        "dequantize_kv_cache": lambda s: rq.resq_dequantize_kv_cache(rows, 128, 16, stream=s),
        "online_hadamard": lambda s: rq.resq_online_hadamard(x, 0, 1024, stream=s),
    }[name]
    want = tensors(call(None))
    side, own = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(own):
        busy = torch.randn(2048, 2048, device=DEV)
        for _ in range(40):
            busy = busy @ busy * 1e-2
        sizes = {t.nbytes for t in want} | {int(rq.lib().resq_sym_eig_workspace_bytes(128))}
        junk = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in sizes if n for _ in range(8)]
        for j in junk:
            j.fill_(85)   # behind what is running
        del junk, j
        got = tensors(call(side))
        torch.cuda.synchronize()
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))
