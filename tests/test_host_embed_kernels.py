"""The embedding's kernels on the CPU, lane by lane (tests/host_sanitize/waves.h), under AddressSanitizer and
UndefinedBehaviorSanitizer: lists, parts, starts, shared memory, partial rows and tables of exactly their sizes; odd sizes,
empty shares, one to three digits, sorts by all tokens and in parts; lanes, waves and blocks in random order, so that a
missing barrier shows as another result.  No GPU."""
import os
import platform
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2111_08617_amd", "csrc")
CLANG = "/opt/rocm/llvm/bin/clang++"
LAUNCHES = "// ---------------------------------------------------------------- launches"

needs = pytest.mark.skipif(not os.path.exists(CLANG) or platform.machine() != "x86_64", reason="needs clang++ and x86-64")


def build_and_run(tmp_path, source, *flags):
    """The driver's run with these kernels, whose launches (which no host compiler reads) are cut off."""
    assert source.count(LAUNCHES) == 1
    (tmp_path / "hip").mkdir()
    (tmp_path / "hip" / "hip_runtime.h").write_text('#include "waves.h"\n#include <cstring>\n')
    (tmp_path / "embed_kernels.inc").write_text(source[:source.index(LAUNCHES)] + "}  // namespace\n}  // namespace cgx\n")
    here = os.path.join(ROOT, "tests", "host_sanitize")
    exe = str(tmp_path / "embed_kernels")
    includes = [f"-I{d}" for d in (tmp_path, here, CSRC, os.path.join(ROOT, "include"))]
    subprocess.run([CLANG, "-std=c++17", "-g", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer", *flags, *includes,
                    os.path.join(here, "embed_kernels.cpp"), os.path.join(CSRC, "cgx_embed.cpp"), "-o", exe], check=True)
    return subprocess.run([exe], capture_output=True, text=True, timeout=600)


def kernels():
    with open(os.path.join(CSRC, "cgx_embed.hip")) as f:
        return f.read()


@needs
def test_every_access_is_inside_and_every_result_right(tmp_path):
    run = build_and_run(tmp_path, kernels(), "-O1", "-fsanitize=address,undefined")
    assert run.returncode == 0, (run.stdout[-2000:], run.stderr[-4000:])
    assert "all checks passed" in run.stdout


@needs
@pytest.mark.parametrize("right, wrong", [
    ("entry[k] = load(at < to ? at : to - 1);", "entry[k] = load(at);"),
    ("            write(first + rank, key, token);\n            __builtin_amdgcn_wave_barrier();", "            write(first + rank, key, token);"),
    ("s.place[k / kDigits][k % kDigits] = 0;\n    __syncthreads();", "s.place[k / kDigits][k % kDigits] = 0;"),
], ids=["a load behind the list", "a wave that does not wait", "a block that does not wait"])
def test_what_it_would_find(tmp_path, right, wrong):
    """Mistakes planted in a copy that only the CPU runs."""
    source = kernels()
    assert source.count(right) == 1
    assert build_and_run(tmp_path, source.replace(right, wrong), "-O0", "-fsanitize=address").returncode != 0
