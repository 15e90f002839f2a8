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
            ('asm volatile("" : "+v"(x));', ""),
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


# ---- attention and norms -------------------------------------------------------------------------------

def prompt(seqs, hq, hk, d, window=0, cap=0.0, scale=None, odd=0, late=1, seed=1):
    return line("prompt", hq, hk, d, window, cap, scale or d ** -0.5, odd, late, seed, len(seqs), [n for s in seqs for n in s])


def prefix(n, lens, hq, hk, d, r, page, order=0, pad=0, window=0, cap=0.0, missing=0, seed=1):
    return line("prefix", hq, hk, d, r, page, order, pad, window, cap, d ** -0.5, missing, seed, n, len(lens), lens)


def check(layer, cases, out, sums):
    for case, got in zip(cases, layer(cases), strict=True):
        assert got[0] <= out and got[1] <= sums, (case, got)


# Scores stay below 8, or so, and are off by less than 2^-20 for their sums of at most 256 products.  Weights are off by 2^-8 of themselves
# (prompts, bf16), values by 2^-11 and weights by 2^-11 of half the codes' range (prefixes, fp16).
PROMPTS, PREFIX, SUMS = 2.0 ** -7.9, 2.0 ** -9.9, 2.0 ** -18


def test_prompts_lengths(layer):
    check(layer, [prompt([(n, 0), (0, 9), (1, n)], 2, 1, 64, late=n % 2) for n in (1, 31, 33, 64, 65, 129, 200)], PROMPTS, SUMS)
    check(layer, [prompt([(30, -20), (5, -5), (9, 0)], 3, 1, 128)], PROMPTS, SUMS)   # more queries than keys


@pytest.mark.parametrize("late", [0, 1])
def test_prompts_widths(layer, late):
    check(layer, [prompt([(40, 30), (3, 0)], 2, 1, d, late=late) for d in (8, 24, 64, 72, 96, 120, 128, 136, 192, 200, 256)], PROMPTS, SUMS)


def test_prompts_parts(layer):
    check(layer, [prompt([(2, 1200)], 2, 1, 64), prompt([(5, 1300), (0, 3), (1, 700)], 1, 1, 128), prompt([(3, 900)], 1, 1, 256, window=300)],
          PROMPTS, SUMS)


def test_prompts_windows_and_caps(layer):
    check(layer, [prompt([(150, 0), (90, 40)], 2, 1, d, window=w, cap=cap, late=w % 2) for d, w, cap in
                  ((64, 1, 0.0), (64, 33, 30.0), (64, 100, 0.5), (128, 64, 0.0), (128, 70, 20.0), (256, 40, 50.0))], PROMPTS, SUMS)


def test_prompts_values_that_are_not_finite(layer):
    check(layer, [prompt([(150, 0), (20, 70)], 1, 1, d, window=w, cap=cap, odd=400) for d, w, cap in ((64, 0, 0.0), (64, 40, 20.0), (136, 90, 0.0))],
          PROMPTS, SUMS)


@pytest.mark.parametrize("d,r", [(8, 0), (8, 8), (40, 16), (64, 8), (72, 4), (96, 12), (128, 16), (128, 128), (200, 100), (256, 252), (256, 0)])
def test_prefix_widths(layer, d, r):
    check(layer, [prefix(n, [0, 7, -1, 20], 2, 1, d, r, page, order, pad=pad, seed=d + r + n) for n, page, order, pad in
                  ((70, 16, 0, 0 if r % 8 else 4), (40, 5, 1, 0 if r % 8 == 0 else 4))], PREFIX, SUMS)


def test_prefix_lengths_windows_caps_and_missing_pages(layer):
    check(layer, [prefix(n, [0, 1, 50, -3], 4, 2, 64, 8, 24, n % 2, window=w, cap=cap, missing=m, seed=n + w) for n, w, cap, m in
                  ((0, 0, 0.0, 0), (1, 0, 0.0, 0), (64, 0, 30.0, 0), (65, 40, 0.0, 3), (300, 150, 20.0, 3), (300, 20, 0.5, 0), (600, 0, 0.0, 3))], PREFIX, SUMS)


def test_prefix_of_more_rows_than_a_workgroup_has(layer):
    check(layer, [prefix(130, [b % 3 for b in range(90)], 3, 1, 8, 8, 16), prefix(70, [1] * 10, 33, 1, 16, 8, 16)], PREFIX, SUMS)


@pytest.mark.parametrize("wide", [0, 1])
def test_norm_widths(layer, wide):
    # a mean square's roundings, at most 64 of 2^-24, and a root: 2^-18 of the result, of which its terms are more; sums of two terms: 2^-22
    check(layer, [line("norm", 3, width, wide, post, gate, alpha, offset, 1e-6, 1, pad, width) for width in (1, 7, 8, 511, 513, 1030, 2049, 4104, 8195, 20001)
                  for post, gate, alpha, offset, pad in ((0, 0, 1, 0, 0), (1, 2, -0.5, 1, 3), (1, 1, 0.22, 0, 1))], 2.0 ** -16, 2.0 ** -17)


# ---- capped scores --------------------------------------------------------------------------------------

@pytest.mark.parametrize("cap", [1e4, 1e6, 1e8, 1.5e38, 3.4e38])
def test_caps_far_above_the_scores_leave_them(layer, cap):
    check(layer, [prompt([(70, 40)], 2, 1, 64, cap=cap), prompt([(3, 900)], 1, 1, 128, cap=cap), prompt([(20, 50)], 1, 1, 136, window=30, cap=cap)],
          PROMPTS, SUMS)
    check(layer, [prefix(130, [0, 30], 2, 1, 64, 8, 16, cap=cap), prefix(130, [0, 3], 2, 1, 256, 32, 16, window=90, cap=cap)], PREFIX, SUMS)


def test_caps_of_any_size(layer):
    caps = (1.2e-38, 1e-20, 1e-3, 1.0, 5.0, 50.0, 500.0)
    check(layer, [prompt([(70, 40)], 2, 1, 64, window=w, cap=cap, scale=1.0) for cap in caps for w in (0, 50)], PROMPTS, SUMS)   # scores of up to 100
    check(layer, [prefix(130, [0, 30], 2, 1, 64, 8, 16, cap=cap) for cap in caps], PREFIX, SUMS)
    check(layer, [prompt([(70, 40)], 2, 1, 64, cap=1.2e-38, scale=scale) for scale in (1e-6, 50.0)], PROMPTS, SUMS)
    check(layer, [prompt([(70, 40)], 2, 1, 64, cap=3.4e38, scale=scale) for scale in (1e-6, 2.0)], PROMPTS, SUMS)
