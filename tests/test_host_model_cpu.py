"""The attention's entry point and kernels in their own source on the CPU (host_model/): every lane of every wavefront, built with the sanitizers for
addresses, alignment and undefined behaviour, on arrays of exactly the size that a call needs.  An access outside of the pages,
the block table, the lengths, the queries, the outputs, the workspace or LDS ends the run."""
import os
import random
import re
import shutil
import subprocess
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
CSRC = ROOT / "paper_2412_14363_amd" / "csrc"
CLANG = shutil.which("clang++", path="/opt/rocm/llvm/bin") or shutil.which("clang++")
SOURCES = ["resq_kv_api.hip", "resq_attend.hip.h", "resq_kv.hip.h", "resq_rope.hip.h", "resq_kv_row.hip.h", "resq_lanes.hip.h", "resq_launch.h",
           "resq_layout.h"]


@pytest.fixture(scope="module")
def attend(tmp_path_factory):
    """runs cases (see host_model/attend.cpp) -> [(outputs' error, log-sum-exps' error)]"""
    if not CLANG:
        pytest.skip("no clang++")
    out = tmp_path_factory.mktemp("model")
    for name in SOURCES:   # as they are but for arrays in LDS of a launch's size, and without unrolling, which only costs time here
        text = re.sub(r"extern __shared__ (?:__attribute__\(\(aligned\(16\)\)\) )?(\w+) (\w+)\[\];", r"\1* \2 = reinterpret_cast<\1*>(model::lds);",
                      (CSRC / name).read_text())
        assert "extern __shared__" not in text
        (out / name).write_text(text.replace("#pragma unroll\n", "\n"))
    exe = out / "attend"
    build = subprocess.run([CLANG, "-std=c++17", "-O0", "-g1", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-Wno-everything",
                            f"-I{ROOT / 'tests' / 'host_model'}", f"-I{out}", f"-I{ROOT / 'include'}",
                            str(ROOT / "tests" / "host_model" / "attend.cpp"), "-o", str(exe)], capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-2000:]

    def run(cases):
        res = subprocess.run([str(exe)], input="\n".join(cases) + "\n", capture_output=True, text=True, timeout=600,
                             env={**os.environ, "ASAN_OPTIONS": "detect_stack_use_after_return=0:detect_leaks=0"})
        assert res.returncode == 0, (cases[len(res.stdout.splitlines())], res.stderr[:3000])
        return [tuple(map(float, line.split())) for line in res.stdout.splitlines()]
    return run


def case(lens, hq, hk, d, r, page, order=0, pad=0, window=0, softcap=0.0, missing=0, seed=1):
    return " ".join(map(str, [len(lens), hq, hk, d, r, page, order, pad, window, softcap, d ** -0.5, missing, seed, *lens]))


def check(attend, cases):
    for c, (off_out, off_lse) in zip(cases, attend(cases), strict=True):
        assert off_out <= 2.0 ** -10 and off_lse <= 2.0 ** -18, (c, off_out, off_lse)


LENS = [0, 1, 15, 16, 17, 31, 33, 64, 127, 129, 300, 0]


def test_attend_pages(attend):
    check(attend, [case(LENS, 4, 2, 128, 16, page, order) for page, order in ((16, 0), (16, 1), (1, 0), (7, 0), (24, 1), (32, 0), (256, 1), (2048, 0))])


@pytest.mark.parametrize("share", [1, 5, 17])
def test_attend_widths(attend, share):
    rng = random.Random(share)
    shapes = [(128, 0), (128, 8), (128, 32), (128, 64), (128, 128), (64, 8), (64, 64), (256, 32), (256, 256), (256, 128), (8, 0), (8, 8), (40, 16),
              (96, 12), (96, 4), (248, 4), (256, 252), (192, 100)]
    check(attend, [case([37, 0, 140, 1], share, 1, d, r, rng.choice((16, 24, 5)), rng.randrange(2), rng.choice((0, 2, 4, 16) if r % 8 else (0, 4, 16)))
                   for d, r in shapes])


def test_attend_windows_caps_and_missing_pages(attend):
    check(attend, [case(LENS + [700], 4, 2, 64, 8, page, order, window=window, softcap=cap, missing=missing, seed=window)
                   for window, cap, missing in ((1, 0.0, 0), (16, 20.0, 3), (31, 0.5, 0), (100, 0.0, 3)) for page, order in ((16, 0), (24, 1))])


def test_attend_cuts(attend):
    # a head in more parts than the join reads at once, several heads in a run, more sequences than a workgroup has threads
    check(attend, [case([1300], 1, 1, 8, 0, 64), case([500, 3, 0, 90], 6, 3, 16, 8, 16), case([1] * 150 + [0] * 120 + [140], 1, 1, 8, 0, 16),
                   case([30] + [0] * 200 + [40] + [0] * 64 + [3], 1, 1, 8, 0, 16),
                   case([0] * 5, 2, 2, 32, 8, 16)])


def test_attend_weights_keep_their_bits(attend):
    # scores are below 8 here, and off by less than 2^-20 for their sums of at most 128 products; weights are off by 2^-17 of half the
    # codes' range (which is no more than a value's size here, zero-point and code apart); fp32 sums are of up to 16 times a value's
    # size, 2^-24 of that for each of a few roundings
    cases = [case([1, 2, 3, 4, 5, 40], 4, 2, d, r, 16) for d, r in ((128, 16), (64, 8), (64, 0), (128, 128), (96, 12))]
    cases.append(case([1, 2, 3, 33], 12, 1, 64, 8, 16))
    for c, (off_out, off_lse) in zip(cases, attend(cases), strict=True):
        assert off_out <= 2.0 ** -16 and off_lse <= 2.0 ** -20, (c, off_out, off_lse)
