"""Which kernels the gated block takes, on the CPU: each that sizes over the operators'
range reach is also taken by a size of the GPU tests that look at every row and column."""
import os
import shutil
import subprocess

import pytest

from test_gpu_extension_tiles import TILE_SHAPES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "tests", "host", "gated_plan_check.cpp")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    out = str(tmp_path_factory.mktemp("gatedplans") / "gated_plan_check")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-Wall", "-Wextra", "-Werror",
           "-I", os.path.join(ROOT, "paper_2609_38198_amd", "csrc"), SRC, "-o", out]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-4000:]
    return out


def taken(driver, shapes):
    lines = []
    for n, d, f, o in shapes:
        lines.append(f"f32 {n} {d} {f} {o}")
        # two planes of H, dG and dU up to this product of sizes
        lines.append(f"{'bf16x2' if n * f * max(d, o) <= 2 ** 25 else 'bf16'} {n} {d} {f} {o}")
    res = subprocess.run([driver, "list"], input="\n".join(lines), capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    return set(res.stdout.splitlines())


def test_every_kernel_in_reach_is_tested(driver):
    res = subprocess.run([driver, "reach"], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    reach = dict(line.split(": ") for line in res.stdout.splitlines())
    assert len(reach) > 60
    have = taken(driver, TILE_SHAPES)
    assert not {k: v for k, v in reach.items() if k not in have}


def test_the_check_notices_a_missing_size(driver):
    kernels = taken(driver, [(64, 64, 64, 64)])
    assert "f32 gate small whole" in kernels and not any(" big " in k for k in kernels)
