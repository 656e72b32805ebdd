"""The tiles of the head's products on the host: launches that fit, and GPU tests that reach every shape."""

import itertools
import os
import shutil
import subprocess

import pytest
import torch

from test_gpu_rows_head import SHAPES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SIDES = {(256, 0): "large", (128, 0): "small", (64, 0): "tiny", (64, 1): "tiny_deep"}


@pytest.fixture(scope="module")
def shapes(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("shapes") / "shapes")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2008_00325_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "rows_head_shapes.cpp"), "-o", exe], check=True, timeout=120)

    def ask(sizes):
        r = subprocess.run([exe], input="\n".join(" ".join(map(str, s)) for s in sizes), capture_output=True, text=True, timeout=60)
        found = [tuple(int(x) for x in line.split()) for line in r.stdout.splitlines()]
        assert r.returncode == 0 and len(found) == len(sizes)
        return found

    return ask


def test_launches_fit(shapes):
    """Fewer than 2^32 work-items: the table's gradient for a piece of at most 2^22 rows, logits of at most 2^27 entries
    of D or 2^24 rows by 256 tokens."""
    sizes = [(m, n, 1, e) for e in (2, 4) for m, n in [*itertools.product((1, 64, 300, 4096, 32768), (1, 1000, 1 << 22)),
                                                       (256, 1 << 24), (1 << 26, 64), (1 << 13, 1 << 14)]]
    for (m, n, _, _), (side, deep) in zip(sizes, shapes(sizes)):
        threads = 512 if side == 256 else 256
        assert -(-m // side) * -(-n // side) * threads < 2**32
        assert not deep or -(-m // side) * -(-n // side) <= 512


def test_gpu_tests_reach_every_shape(shapes):
    """For each product (logits, rows' gradient, table's gradient) and both widths of elements."""
    asked, seen = [], {}
    for n, rows, cols, dtype in SHAPES:
        elem = dtype.itemsize
        parts = 2 if elem == 2 and n <= 256 else 1
        steps = -(-(-(-rows // 256) * 256) // (128 // elem))
        if n > 64:
            asked.append(("logits", elem, (rows, n, 1, elem)))
        if n * parts > 64:
            asked.append(("rows", elem, (cols, n * parts, max(1, steps // (2 if elem == 4 else 4)), elem)))
        asked.append(("table", elem, (cols, rows, 1, elem)))
    for (name, elem, _), found in zip(asked, shapes([a[2] for a in asked])):
        seen.setdefault((name, elem), set()).add(SIDES[found])
    for key, value in seen.items():
        assert value == set(SIDES.values()), (key, value)
    few = {(n <= 32, dtype.itemsize) for n, rows, cols, dtype in SHAPES if n <= 64 and rows * cols * dtype.itemsize >= 8 << 20}
    assert few == {(True, 2), (True, 4), (False, 2), (False, 4)}
    assert torch.float16 in {s[3] for s in SHAPES}
