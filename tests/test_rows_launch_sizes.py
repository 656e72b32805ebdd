"""The norm's grids on the host: fewer than 2^32 work-items however many rows, and never
fewer than four workgroups for each of 256 CUs where there is work for them."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_norm_grids(tmp_path):
    exe = str(tmp_path / "sizes")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2008_00325_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "rows_launch_sizes.cpp"), "-o", exe], check=True, timeout=120)
    asked = [(w, c, t) for w in (1, 3, 1000, 1023, 1024, 4096, 10**6, 2**24, 2**24 + 1, 2**31 - 1) for t in (64, 256, 320, 512, 1024)
             for c in (8, 512, 4096)]
    r = subprocess.run([exe], input="\n".join(f"{w} {c} {t}" for w, c, t in asked), capture_output=True, text=True, timeout=60)
    grids = [int(x) for x in r.stdout.split()]
    assert r.returncode == 0 and len(grids) == len(asked)
    for (w, _, t), g in zip(asked, grids):
        assert 1 <= g <= w and g * t < 2**32
        assert g >= min(w, 1024)
