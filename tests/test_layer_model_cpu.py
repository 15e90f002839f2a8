"""The entry points around a layer's products and their kernels in their own source on the CPU (host_model/), every lane of every wavefront, built with
the sanitizers for addresses, alignment and undefined behaviour, on arrays of exactly the size that a call needs.  Loads straight to LDS arrive at once in
some cases, and only where the kernel waits for them in others."""
import os
import re
import subprocess

import pytest

from test_host_model_cpu import CLANG, CSRC, ROOT, SOURCES

LAYER_SOURCES = [*SOURCES, "resq_layer_api.hip", "resq_norm.hip.h", "resq_flash.hip.h", "resq_prompts.hip.h", "resq_prefix.hip.h"]
MODEL = ROOT / "tests" / "host_model"


def replaced(text, pairs):
    for old, new in pairs:
        assert old in text, old
        text = text.replace(old, new)
    return text


def source(name):
    """as it is but for arrays in LDS of a launch's size, unrolling, which only costs time here, and what is not C++"""
    text = re.sub(r"extern __shared__ (?:__attribute__\(\(aligned\(16\)\)\) )?(\w+) (\w+)\[\];", r"\1* \2 = reinterpret_cast<\1*>(model::lds);",
                  (CSRC / name).read_text())
    assert "extern __shared__" not in text
    text = re.sub(r"#pragma unroll( \d+)?\n", "\n", text)
    if name == "resq_layer_api.hip":   # (one file with the other entry points here)
        text = text.replace("kInt32Max", "kLayerInt32Max")
    if name == "resq_flash.hip.h":
        wait = lambda n: "model::wait_but(%s); model::barrier();" % n
        text = replaced(text, [
            ("#define FlashLds __attribute__((address_space(3)))", "#define FlashLds"),
            (r'asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");',
             "model::fetch(lds, base, off);"),
            (r'asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");', wait(0)),
            (r'asm volatile("s_waitcnt lgkmcnt(0)\n\ts_setprio 0\n\ts_barrier" ::: "memory");', "model::barrier();"),
            (r'asm volatile("s_waitcnt lgkmcnt(0)\n\ts_setprio 3\n\ts_barrier" ::: "memory");', "model::barrier();"),
            (r'asm volatile("s_waitcnt vmcnt(%0)\n\ts_setprio 3\n\ts_barrier" ::"n"(LATER) : "memory");', wait("LATER"))])
        assert "asm volatile" not in text
    return text


@pytest.fixture(scope="module")
def layer(tmp_path_factory):
    """runs cases (see host_model/layer.cpp) -> [(outputs' error, sums' error)]"""
    if not CLANG:
        pytest.skip("no clang++")
    out = tmp_path_factory.mktemp("layer")
    for name in LAYER_SOURCES:
        (out / name).write_text(source(name))
    (out / "hip").mkdir()
    (out / "hip" / "hip_ext.h").write_text((MODEL / "hip" / "hip_ext.h").read_text())
    (out / "hip" / "hip_runtime.h").write_text(replaced((MODEL / "hip" / "hip_runtime.h").read_text(), [   # workgroups of up to 1024, LDS low in memory
        ("kMaxThreads = 256", "kMaxThreads = 1024"),
        ("\nnamespace model {\n", "\nnamespace model {\ninline int low_lds(void**, size_t, size_t);\ninline void low_lds_done(void*);\n"),
        ("posix_memalign(&p, 16, lds_bytes)", "low_lds(&p, 16, lds_bytes)"), ("free(lds)", "low_lds_done(lds)")]))
    exe = out / "layer"
    build = subprocess.run([CLANG, "-std=c++17", "-O0", "-mf16c", "-g1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wno-everything",
                            f"-I{out}", f"-I{MODEL}", f"-I{ROOT / 'include'}", str(MODEL / "layer.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-2000:]

    def run(cases):
        res = subprocess.run([str(exe)], input="\n".join(cases) + "\n", capture_output=True, text=True, timeout=600,
                             env={**os.environ, "ASAN_OPTIONS": "detect_stack_use_after_return=0:detect_leaks=0"})
        assert res.returncode == 0, (cases[len(res.stdout.splitlines())], res.stderr[:3000])
        return [tuple(map(float, line.split())) for line in res.stdout.splitlines()]
    return run


def line(*parts):
    return " ".join(" ".join(map(str, p)) if isinstance(p, (list, tuple)) else str(p) for p in parts)


# ---- the search for a workgroup's rows ----------------------------------------------------------------

@pytest.mark.parametrize("waves", [4, 8])
def test_each_workgroup_finds_its_rows(layer, waves):
    """Lengths that do not decrease: each tile of rows is found once, whatever stands between them."""
    cases = []
    for share, lens in ((1, [300, 0, 1, 5, 900, 0]), (7, [0, 40, 33, 0, 0, 256]), (4, [64] * 40), (3, [0, 1, 0, 2] * 100), (1, [1 << 30])):
        cu = [sum(lens[:i]) for i in range(len(lens) + 1)]
        cases.append(line("tiles", waves, len(lens), share, cu[-1], cu[-1], cu, cu))
    for got, case in zip(layer(cases), cases, strict=True):
        assert got[0] == 0, (case, got)


@pytest.mark.parametrize("waves", [4, 8])
@pytest.mark.parametrize("batch,share,tokens,pattern", [
    (3, 4, 40, [30, 10, 40, 5]), (65535, 8, 1 << 23, [0, 1 << 23]), (65535, 1, 1 << 30, [0, 1 << 30]), (65535, 2, 1 << 29, [0, 1 << 29, 1 << 28, -5]),
    (600, 64, 1 << 24, [1 << 24, 0, 7, 1 << 30]), (65535, 1, 16700000, [16700000, 0, 3])])
def test_lengths_that_decrease_stay_inside_of_the_tensors(layer, waves, batch, share, tokens, pattern):
    """Their results are unspecified; rows and keys of a workgroup are some of the tensors' all the same."""
    got, = layer([line("tiles", waves, batch, share, tokens, tokens // 2, pattern, pattern[::-1])])
    assert got[0] == 0, got
