"""Overlap of the token-row calls' arrays (no GPU): refused exactly where they share an element, for
matrices of one pitch and for a single row among another matrix's."""

import itertools

import pytest

from paper_2008_00325_amd import umap_layout as U
from paper_2008_00325_amd import umap_rows as R

A, FAR, COLS = 1 << 40, 1 << 50, 3   # addresses that are only compared


def elements(first, n, stride):
    return {first + i * stride + c for i in range(n) for c in range(COLS)}


def y_is_refused(x, y):
    """Each call is refused before anything runs: for y, or else for h, which lies on the weight."""
    X, Y = (R.umap_rows(A + 4 * first, None, n, stride, COLS, R.UMAP_F32, 0, 0) for first, n, stride in (x, y))
    h = R.umap_rows(FAR, None, y[1], COLS, COLS, R.UMAP_F32, 0, 0)
    rc = R.lib().umap_rows_norm(X, 2 * FAR, R.UMAP_I32, 1.0, None, h, FAR, R.UMAP_F32, 1e-6, Y, None)
    text = U.umap_layout_last_error()
    assert rc == U.UMAP_E_INVAL and text.startswith(("y overlaps", "h overlaps")), text
    return text.startswith("y")


@pytest.mark.parametrize("n,m", [(4, 4), (2, 5), (1, 4), (4, 1), (1, 1)])
@pytest.mark.parametrize("stride", [3, 5, 6, 7, 9])
def test_refused_where_an_element_is_shared(n, m, stride):
    seen = set()
    for first, single in itertools.product(range(-40, 41), (3, 100)):
        # a single row's own stride means nothing
        x, y = ((at, k, stride if k > 1 else single) for at, k in ((0, n), (first, m)))
        share = bool(elements(*x) & elements(*y))
        assert y_is_refused(x, y) == share, (x, y)
        seen.add(share)
    assert seen == {True, False}
