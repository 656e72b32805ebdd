"""Boundary of the token-row operators that needs no GPU: what the header declares is
exported and bound, and every invalid argument is refused before any HIP call."""

import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2008_00325_amd import umap_layout as U
from paper_2008_00325_amd import umap_rows as R

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "umap_rows.h")
A = 1 << 40   # addresses that are only compared


def test_every_declared_function_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(umap_rows_\w+)\s*\(", text)))
    assert sorted(R.EXPORTS) == names
    for name in names:
        assert hasattr(R.lib(), name)


def test_constants_match_header():
    for name, value in re.findall(r"#define (UMAP_\w+) (\d+)", open(HEADER).read()):
        assert getattr(R, name) == int(value)


def test_struct_has_the_header_s_layout():
    assert ctypes.sizeof(R.umap_rows) == 48
    assert [R.umap_rows.data.offset, R.umap_rows.scales.offset, R.umap_rows.rows.offset, R.umap_rows.stride.offset,
            R.umap_rows.cols.offset, R.umap_rows.type.offset, R.umap_rows.group.offset] == [0, 8, 16, 24, 32, 36, 40]


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not available")
def test_header_is_plain_c(tmp_path):
    src = tmp_path / "client.c"
    src.write_text("""#include "umap_rows.h"
_Static_assert(sizeof(umap_rows) == 48, "size");
int main(void)
{
    umap_rows m = {0, 0, 0, 8, 8, UMAP_BF16, 0, 0};
    return umap_rows_lookup(&m, 0, UMAP_I64, 1.0f, &m, 0) + (int)umap_rows_norm_grad_workspace(0, 8);
}
""")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", "-fsyntax-only", "-I", os.path.dirname(HEADER),
                    str(src)], check=True, timeout=60)


def rows(at, n=10, cols=16, type=R.UMAP_F32, stride=None, scales=None, group=0, reserved=0):
    return R.umap_rows(at, scales, n, cols if stride is None else stride, cols, type, group, reserved)


def refused(rc, part):
    assert rc == U.UMAP_E_INVAL and part in U.umap_layout_last_error(), (rc, U.umap_layout_last_error())


BAD = [
    (dict(type=5), "element type"),
    (dict(type=-1), "element type"),
    (dict(cols=0), "cols"),
    (dict(cols=-3), "cols"),
    (dict(cols=(1 << 20) + 1), "cols"),
    (dict(n=-1), "rows"),
    (dict(stride=15), "stride"),
    (dict(stride=-16), "stride"),
    (dict(stride=1 << 60), "too many"),
    (dict(n=1 << 60), "too many"),
    (dict(reserved=1), "reserved"),
    (dict(at=0), "NULL"),
    (dict(at=A + 2), "aligned"),
    (dict(group=32), "8-bit"),
    (dict(scales=A), "8-bit"),
    (dict(type=R.UMAP_I8), "need scales"),
    (dict(type=R.UMAP_I8, scales=A + (1 << 30), group=16), "group"),
    (dict(type=R.UMAP_F8, scales=A + 2, group=32), "not aligned"),
]


@pytest.mark.parametrize("change,part", BAD)
def test_lookup_refuses_bad_tables(change, part):
    bad = {"at": A, **change}
    refused(R.lib().umap_rows_lookup(rows(**bad), A + (1 << 34), R.UMAP_I32, 1.0, rows(2 * A, cols=bad.get("cols", 16)), None), part)


@pytest.mark.parametrize("change,part", [b for b in BAD if "type" not in b[0]] + [(dict(type=R.UMAP_I8), "element type"),
                                                                              (dict(stride=0), "stride")])
def test_lookup_refuses_bad_outputs(change, part):
    bad = {"at": A, **change}
    refused(R.lib().umap_rows_lookup(rows(2 * A, cols=max(1, bad.get("cols", 16))), A + (1 << 60), R.UMAP_I32, 1.0, rows(**bad), None), part)


def test_lookup_refuses():
    f = R.lib().umap_rows_lookup
    t, o, i = rows(A), rows(2 * A), 3 * A
    refused(f(None, i, R.UMAP_I32, 1.0, o, None), "table must not be NULL")
    refused(f(t, i, R.UMAP_I32, 1.0, None, None), "out must not be NULL")
    refused(f(t, i, 3, 1.0, o, None), "id_type")
    refused(f(t, i + 4, R.UMAP_I64, 1.0, o, None), "ids are not aligned")
    refused(f(t, i, R.UMAP_I32, float("nan"), o, None), "scale")
    refused(f(t, i, R.UMAP_I32, float("inf"), o, None), "scale")
    refused(f(t, i, R.UMAP_I32, 1.0, rows(2 * A, cols=17), None), "cols")
    refused(f(t, None, 0, 1.0, rows(2 * A, n=11), None), "out has 11 rows")
    refused(f(t, i, R.UMAP_I32, 1.0, rows(A + 64), None), "overlaps")
    refused(f(t, 2 * A + 4, R.UMAP_I32, 1.0, o, None), "overlaps")
    refused(f(rows(A, type=R.UMAP_I8, scales=2 * A + 100), i, R.UMAP_I32, 1.0, o, None), "overlaps")
    # interleaved columns that meet in one element
    refused(f(rows(A, stride=40), i, R.UMAP_I32, 1.0, rows(A + 15 * 4, stride=40), None), "overlaps")
    refused(f(rows(A, stride=40), i, R.UMAP_I32, 1.0, rows(A + 25 * 4, stride=40), None), "overlaps")
    assert f(t, i, R.UMAP_I32, 1.0, rows(0, n=0), None) == U.UMAP_OK   # nothing to do


def test_lookup_grad_refuses():
    L = R.lib()
    need = L.umap_rows_lookup_grad_workspace(10, 20, 16)
    assert need > 0
    ok = dict(d=rows(A), i=3 * A, it=R.UMAP_I32, s=1.0, g=rows(2 * A, n=20), a=0, w=4 * A, wb=need)

    def f(**kw):
        v = {**ok, **kw}
        return L.umap_rows_lookup_grad(v["d"], v["i"], v["it"], v["s"], v["g"], v["a"], v["w"], v["wb"], None)

    refused(f(d=None), "dout must not be NULL")
    refused(f(g=None), "grad must not be NULL")
    refused(f(i=None), "ids must not be NULL")
    refused(f(it=R.UMAP_F32), "id_type")
    refused(f(s=float("-inf")), "scale")
    refused(f(a=2), "accumulate")
    refused(f(w=None), "workspace of 0 bytes")
    refused(f(wb=need - 1), "workspace of")
    refused(f(w=4 * A + 8), "aligned to 16")
    refused(f(d=rows(A, type=R.UMAP_I8, scales=A)), "element type")
    refused(f(g=rows(2 * A, n=20, type=R.UMAP_F8, scales=A)), "element type")
    refused(f(g=rows(2 * A, n=20, cols=15)), "cols")
    refused(f(g=rows(2 * A, n=2**31 - 1)), "rows of grad")
    refused(f(d=rows(A, n=2**31)), "rows of dout")
    refused(f(g=rows(A + 4, n=20)), "grad overlaps")
    refused(f(g=rows(3 * A - 32, n=20)), "grad overlaps")
    refused(f(w=A + 16), "workspace overlaps")
    refused(f(w=2 * A + 16), "overlaps")
    for bad in ((-1, 20, 16), (2**31, 20, 16), (10, -1, 16), (10, 2**31, 16), (10, 20, 0), (10, 20, 2**20 + 1)):
        assert L.umap_rows_lookup_grad_workspace(*bad) == U.UMAP_E_INVAL
    assert f(d=rows(0, n=0), i=None, a=1) == U.UMAP_OK


def test_norm_refuses():
    L = R.lib()
    ok = dict(x=rows(A), i=None, it=0, s=1.0, r=rows(2 * A), h=rows(3 * A), w=4 * A, wt=R.UMAP_F32, e=1e-6, y=rows(5 * A))

    def f(**kw):
        v = {**ok, **kw}
        return L.umap_rows_norm(v["x"], v["i"], v["it"], v["s"], v["r"], v["h"], v["w"], v["wt"], v["e"], v["y"], None)

    refused(f(x=None), "x must not be NULL")
    refused(f(y=None), "y must not be NULL")
    refused(f(x=rows(A, type=R.UMAP_I8, scales=6 * A)), "element type")
    refused(f(x=rows(A, cols=32769), y=rows(5 * A, cols=32769)), "cols")
    refused(f(y=rows(5 * A, cols=17)), "cols")
    refused(f(y=rows(5 * A, n=11)), "rows")
    refused(f(r=rows(2 * A, n=9)), "residual has 9 rows")
    refused(f(r=rows(2 * A, type=R.UMAP_BF16)), "residual must have x's type")
    refused(f(h=rows(3 * A, type=R.UMAP_F16)), "h must have x's type")
    refused(f(h=rows(3 * A, n=11)), "h has 11 rows")
    refused(f(w=4 * A + 2), "weight is not aligned")
    refused(f(wt=R.UMAP_I8), "weight_type")
    refused(f(e=-1e-6), "eps")
    refused(f(e=float("nan")), "eps")
    refused(f(s=float("nan")), "scale")
    refused(f(i=6 * A, it=7), "id_type")
    refused(f(y=rows(A)), "y overlaps")
    refused(f(y=rows(5 * A, type=R.UMAP_I8, scales=5 * A + 64)), "y overlaps")
    refused(f(y=rows(5 * A, type=R.UMAP_I8, scales=2 * A + 64)), "scales overlaps")
    refused(f(h=rows(A + 64)), "h overlaps")
    refused(f(h=rows(A, stride=17)), "h overlaps")
    refused(f(i=6 * A, it=R.UMAP_I32, h=rows(A)), "h overlaps")   # gathered rows are read after others are written
    refused(f(h=rows(4 * A)), "h overlaps")
    assert f(x=rows(0, n=0), y=rows(0, n=0), r=None, h=None) == U.UMAP_OK


def test_norm_grad_refuses():
    L = R.lib()
    need = L.umap_rows_norm_grad_workspace(10, 16)
    assert need > 0
    ok = dict(dy=rows(A), h=rows(2 * A), dh=rows(3 * A), w=4 * A, wt=R.UMAP_F32, e=1e-6, dx=rows(5 * A), dw=6 * A,
              ws=7 * A, wb=need)

    def f(**kw):
        v = {**ok, **kw}
        return L.umap_rows_norm_grad(v["dy"], v["h"], v["dh"], v["w"], v["wt"], v["e"], v["dx"], v["dw"], v["ws"], v["wb"], None)

    for name in ("dy", "h", "dx"):
        refused(f(**{name: None}), f"{name} must not be NULL")
    refused(f(h=rows(2 * A, n=9)), "h has 9 rows")
    refused(f(dx=rows(5 * A, cols=15)), "dx has 15 cols")
    refused(f(dh=rows(3 * A, type=R.UMAP_BF16)), "one type")
    refused(f(dy=rows(A, n=2**31)), "rows must be")
    refused(f(e=float("inf")), "eps")
    refused(f(wt=9), "weight_type")
    refused(f(dw=6 * A + 1), "dweight is not aligned")
    refused(f(ws=None), "workspace of 0 bytes")
    refused(f(wb=need - 1), "workspace of")
    refused(f(ws=7 * A + 4), "aligned to 16")
    refused(f(dx=rows(2 * A)), "dx overlaps")
    refused(f(dx=rows(A + 64)), "dx overlaps")
    refused(f(dw=A), "dweight overlaps")
    refused(f(dw=5 * A + 64), "overlaps")
    refused(f(ws=2 * A), "workspace overlaps")
    refused(f(ws=5 * A), "overlaps")
    for bad in ((-1, 16), (2**31, 16), (10, 0), (10, 32769)):
        assert L.umap_rows_norm_grad_workspace(*bad) == U.UMAP_E_INVAL
    assert f(dy=rows(0, n=0), h=rows(0, n=0), dh=None, dx=rows(0, n=0), dw=None) == U.UMAP_OK


def test_binding_refuses():
    cpu = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU tensor"):
        R.umap_rows_lookup(cpu, None, cpu)
    with pytest.raises(ValueError, match="must not hold"):
        R.umap_rows_lookup(cpu.double(), None, cpu)
    with pytest.raises(U.UmapLayoutError, match="cols"):
        R.umap_rows_norm_grad_workspace(4, 0)
    with pytest.raises(U.UmapLayoutError, match="rows of grad"):
        R.umap_rows_lookup_grad_workspace(4, -1, 8)
