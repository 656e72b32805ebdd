"""The limits that the token-row header states are those that the library enforces (no GPU)."""

import os
import re

import pytest

from paper_2008_00325_amd import umap_layout as U
from paper_2008_00325_amd import umap_rows as R

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "umap_rows.h")
A = 1 << 40   # addresses that are only compared


def stated(call, argument):
    """The largest number of rows that the call's comment allows the argument."""
    text = open(HEADER).read()
    comment = next(c for c in re.findall(r"/\*(.*?)\*/", text, flags=re.S) if f"{call} --" in c)
    comment = re.sub(r"\n \*", "\n", comment)
    # an argument's text goes on until the next argument's line
    entry = re.search(rf"^ {{3}}{argument} {{2}}.*?(?=^ {{3}}\w|^\s*$|\Z)", comment, flags=re.S | re.M).group(0)
    power, less = re.search(r"rows\s+<\s+2\^(\d+)(?: - (\d+))?", entry).groups()
    return 2**int(power) - int(less or 0) - 1


def rows(at, n):
    return R.umap_rows(at, None, n, 0, 16, R.UMAP_F32, 0, 0)


def out(at, n):
    return R.umap_rows(at, None, n, 16, 16, R.UMAP_F32, 0, 0)


def lookup_grad(dout=10, grad=10):
    return R.lib().umap_rows_lookup_grad(rows(A, dout), 1 << 60, R.UMAP_I32, 1.0, out(1 << 50, grad), 0, None, 0, None)


def norm(y):
    return R.lib().umap_rows_norm(rows(A, y), None, 0, float("nan"), None, None, None, 0, 1e-6, out(1 << 50, y), None)


def norm_grad(dy):
    return R.lib().umap_rows_norm_grad(rows(A, dy), rows(2 * A, dy), None, None, 0, -1.0, out(1 << 50, dy), None, None, 0, None)


@pytest.mark.parametrize("call,argument,refused", [
    ("umap_rows_lookup_grad", "dout", lambda n: lookup_grad(dout=n)),
    ("umap_rows_lookup_grad", "grad", lambda n: lookup_grad(grad=n)),
    ("umap_rows_norm", "y", norm),
    ("umap_rows_norm_grad", "dy, h", norm_grad),
])
def test_rows_up_to_the_stated_limit(call, argument, refused):
    """Each call is refused: for the number of rows beyond the limit, for another argument up to it."""
    most = stated(call, argument)
    assert refused(most + 1) == U.UMAP_E_INVAL and "rows" in U.umap_layout_last_error()
    assert refused(most) == U.UMAP_E_INVAL and not re.search(r"rows .*must be", U.umap_layout_last_error())


def test_workspaces_have_the_same_limits():
    L = R.lib()
    for argument, size in (("dout", lambda n: L.umap_rows_lookup_grad_workspace(n, 10, 16)),
                           ("grad", lambda n: L.umap_rows_lookup_grad_workspace(10, n, 16))):
        most = stated("umap_rows_lookup_grad", argument)
        assert size(most) > 0 and size(most + 1) == U.UMAP_E_INVAL
    most = stated("umap_rows_norm_grad", "dy, h")
    assert L.umap_rows_norm_grad_workspace(most, 16) > 0 and L.umap_rows_norm_grad_workspace(most + 1, 16) == U.UMAP_E_INVAL
