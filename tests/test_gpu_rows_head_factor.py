"""The product dscale * scale * dloss, where two of its factors leave fp32's range and all three do not."""

import pytest
import torch

from paper_2008_00325_amd import umap_rows as R
from test_gpu_rows import DEV, F32, FLOATS
from test_gpu_rows_head import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seed():
    torch.manual_seed(17)
    yield
    torch.cuda.synchronize()


def both(case, lse, dloss, dscale):
    dh, dw = torch.empty_like(case.H), torch.empty_like(case.W)
    case.grad(lse, dh, dw, dloss, dscale)
    return dh, dw


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("n,k", [(60, 0), (60, 6), (300, 0), (9000, 2)])
def test_large_and_small_factors_cancel(n, k, dtype):
    """Powers of two change no digit: the bits are those of ordinary factors."""
    case = Case(n, 300, 40, dtype, k=k, lean=3.0)
    case.H, case.W, case.scale = (case.H.float() / 4).to(dtype), (case.W.float() / 4).to(dtype), 16.0
    lse = case.loss()[1]
    w = torch.rand(n, device=DEV) + 0.25
    want = both(case, lse, w, 2.0**4)
    for power in (124, 127):   # dscale * scale is 2^128 and more, the weight of a row 2^8 w
        found = both(case, lse, w * 2.0 ** (4 - power), 2.0**power)
        assert all(torch.equal(a, b) for a, b in zip(found, want)), power


def test_a_small_product_keeps_its_digits():
    """dscale * scale is 1.2345 x 2^-130, the gradients, whose vectors are larger, are ordinary numbers."""
    case = Case(50, 200, 40, F32)
    case.W, case.H, case.scale = case.W * 2.0**40, case.H * 2.0**-10, 2.0**-30
    lse = case.loss()[1]
    want = both(case, lse, None, 1.2345 * 2.0**20)
    small = both(case, lse, None, 1.2345 * 2.0**-100)
    assert torch.equal(small[0], want[0] * 2.0**-120)


@pytest.mark.parametrize("weighted", [False, True])
def test_a_large_product_of_rows_without_part(weighted):
    """dscale * scale beyond fp32's range is times nothing where no row takes part, or there is none."""
    case = Case(20, 50, 16, F32, absent=2.0)
    case.scale = 2.0**60
    case.W *= 2.0**-60
    lse = case.loss()[1]
    w = torch.rand(20, device=DEV) if weighted else None
    dh, dw = both(case, lse, w, 2.0**100)
    assert not bool(dh.any()) and not bool(dw.any())
    none = torch.empty(0, device=DEV)
    work = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    dw = torch.ones_like(case.W)
    R.umap_rows_cross_entropy_grad(case.H[:0], case.W, case.tokens[:0], none, work, dtable=dw, dloss=none if weighted else None,
                                   dscale=2.0**100, scale=case.scale)
    assert not bool(dw.any())
