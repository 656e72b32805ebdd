"""The tiles of the head's logits on the host: those that there are for a type, all of them reached by the GPU tests."""

import os
import shutil
import subprocess

import pytest

from test_gpu_rows_head import SHAPES
from test_rows_head_shapes import ROOT, SIDES


def shapes(tmp_path, sizes):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "shapes")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2008_00325_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "rows_logits_shapes.cpp"), "-o", exe], check=True, timeout=120)
    r = subprocess.run([exe], input="\n".join(" ".join(map(str, s)) for s in sizes), capture_output=True, text=True, timeout=60)
    found = [SIDES[tuple(int(x) for x in line.split())] for line in r.stdout.splitlines()]
    assert r.returncode == 0 and len(found) == len(sizes)
    return found


def test_gpu_tests_reach_every_tile_of_the_logits(tmp_path):
    asked = [(rows, n, dtype.itemsize) for n, rows, _, dtype in SHAPES if n > 64]
    seen = {2: set(), 4: set()}
    for (_, _, elem), side in zip(asked, shapes(tmp_path, asked)):
        seen[elem].add(side)
    assert seen[2] == {"large", "small", "tiny", "tiny_deep"}
    assert seen[4] == {"small", "tiny", "tiny_deep"}


def test_fp32_has_no_large_tile(tmp_path):
    sizes = [(rows, n) for rows in (65, 1000, 4100, 32_000, 128_000, (1 << 26) - 1) for n in (65, 300, 3100, 8192, (1 << 24) - 1)]
    assert "large" not in shapes(tmp_path, [(*s, 4) for s in sizes])
    assert "large" in shapes(tmp_path, [(*s, 2) for s in sizes])
