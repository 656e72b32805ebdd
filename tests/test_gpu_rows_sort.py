"""Gradient of the lookup at the numbers of ids between which its sort changes launches."""

import pytest
import torch

from test_gpu_rows import BF16, check_grad, rand, zipf

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1024, 1025, 4096, 4097, 8192, 8193, 131_072, 131_073, 524_288, 524_289, 1_048_575, 1_048_576, 1_048_577])
@pytest.mark.parametrize("rows", [300, 70_000])
def test_grad_on_both_sides_of_the_sorts_bounds(n, rows):
    torch.manual_seed(n)
    check_grad(rand(n, 5, BF16), zipf(n, rows, torch.int32), rows)
