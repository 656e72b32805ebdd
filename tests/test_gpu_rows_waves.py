"""Norm gradient with dweight on both sides of the widths between which its workgroups change in number."""

import pytest

from test_gpu_rows import BF16, F32, check_norm_grad, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [7, 8, 47, 48, 49, 64, 65, 128, 129, 256, 257, 512, 513, 1024, 1025])
@pytest.mark.parametrize("n", [1, 31, 33, 513, 1025, 20_000])
def test_norm_grad_on_both_sides_of_the_widths(dim, n):
    n = min(n, 3_000_000 // dim)
    check_norm_grad(rand(n, dim, BF16), rand(n, dim, BF16), rand(1, dim, F32)[0])
