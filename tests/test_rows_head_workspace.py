"""The head's workspaces stay within what the header says of them."""

import itertools

import pytest

from paper_2008_00325_amd import umap_rows as R

MB = 1 << 20
SIZES = list(itertools.product((1, 64, 257, 8192, 131_072, (1 << 24) - 1), (1, 300, 32_003, 128_000, 5_000_000, (1 << 26) - 1),
                               (1, 64, 1001, 4096, 32_768), (R.UMAP_F32, R.UMAP_BF16)))


def common(n, rows, cols, type_):
    elem, wide = (4 if type_ == R.UMAP_F32 else 2), -(-cols // 64) * 64
    return elem, wide, min(max(128 * MB, 256 * wide * elem), (rows + 255) * wide * elem)


@pytest.mark.parametrize("k", [1, 20, 256])
def test_sizes_are_those_of_the_header(k):
    L = R.lib()
    for n, rows, cols, type_ in SIZES:
        elem, wide, table = common(n, rows, cols, type_)
        need = L.umap_rows_distill_workspace(n, rows, cols, k, type_)
        assert 0 < need <= n * wide * elem + table + max(128 * MB, 32 * (rows + 63)) + 4 * n + 1024, (n, rows, cols, type_)
        parts = 2 if elem == 2 and n <= 256 else 1
        need = L.umap_rows_distill_grad_workspace(n, rows, cols, k, type_)
        d, sums = max(256 * MB, n * parts * 256 * elem), max(72 * MB, n * parts * (cols + 3) * 4)
        assert 0 < need <= 2 * n * parts * wide * elem + table + d + sums + n * (100 + 8 * k) + 4096, (n, rows, cols, type_)
