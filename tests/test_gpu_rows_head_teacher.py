"""A teacher's shares: empty places at every scale, products beyond fp32's range, and the precision of small shares."""

import math

import pytest
import torch

from paper_2008_00325_amd import umap_rows as R
from rows_reference import E32
from test_gpu_rows import DEV, F32, FLOATS
from test_gpu_rows_head import F64, Case, near

pytestmark = pytest.mark.gpu


def outputs(case):
    loss, lse = case.loss()
    dh, dw = torch.empty_like(case.H), torch.empty_like(case.W)
    case.grad(lse, dh, dw, dscale=0.25)
    return loss, lse, dh, dw


@pytest.fixture(autouse=True)
def _seed():
    torch.manual_seed(13)
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("teacher", FLOATS)
@pytest.mark.parametrize("scale", [0.0, -0.5, 1.0])
@pytest.mark.parametrize("n,k", [(40, 5), (300, 70), (2100, 3)])
def test_places_of_minus_infinity_are_empty(n, k, scale, teacher):
    """At every scale, 0 and negative ones among them: the bits of the same call whose places have no token."""
    case = Case(n, 200, 40, F32, k=k, teacher=teacher, teacher_scale=scale)
    empty = torch.rand(n, k, device=DEV) < 0.3
    empty[7] = True
    tokens, logits = case.tokens, case.A
    case.A = logits.masked_fill(empty, -math.inf)
    found = outputs(case)
    case.A, case.tokens = logits, tokens.masked_fill(empty, -1)
    want = outputs(case)
    assert all(bool(torch.isfinite(x).all()) for x in found)
    assert float(found[0][7]) == 0 and not bool(found[2][7].any())
    assert all(torch.equal(a, b) for a, b in zip(found, want))
    if scale == 0:   # alike, whatever the logits
        case.A = torch.zeros_like(logits)
        assert all(torch.equal(a, b) for a, b in zip(outputs(case), want))


def test_the_largest_logits_at_a_scale_of_0_are_alike():
    case = Case(30, 100, 24, F32, k=4, absent=0.0, teacher_scale=0.0)
    case.A = torch.tensor([3e38, -3e38, 1e38, -1e38], device=DEV).expand(30, 4).contiguous()
    found = outputs(case)
    case.A = torch.zeros_like(case.A)
    assert all(torch.equal(a, b) for a, b in zip(found, outputs(case)))


@pytest.mark.parametrize("scale", [8.0, -8.0])
def test_products_beyond_the_range(scale):
    """Finite logits and scales whose product is none: the largest product has all of the row."""
    case = Case(30, 100, 24, F32, k=4, absent=0.0, teacher_scale=scale)
    case.tokens[:, 1:] = (case.tokens[:, :1] + torch.arange(1, 4, device=DEV)) % 100
    case.A = torch.tensor([3e38, -3e38, 1e38, -1e38], device=DEV).expand(30, 4).contiguous()
    loss, lse, dh, dw = outputs(case)
    one = Case(30, 100, 24, F32)
    one.H, one.W, one.tokens = case.H, case.W, case.tokens[:, 0 if scale > 0 else 1].contiguous()
    want = outputs(one)
    # q is 1 and 0 in both calls; the loss's own logit is a dot product, of which the order may differ
    near(loss, want[0].to(F64), 1e-5 + 0 * want[0].to(F64), "loss")
    assert torch.equal(lse, want[1])
    for got, ref in ((dh, want[2]), (dw, want[3])):
        near(got, ref.to(F64), 1e-5 + 0 * ref.to(F64), "gradient")


def test_small_shares_are_as_exact_as_fp32():
    """A table of unit vectors and rows whose probability of the teacher's tokens is 0 (a logit of -200): dh is -q.  A share is off
    by 2 E32 of its exponential, 2 of the others' and 6 of their sum in a tree of 64, 1 of the quotient, and 2 where D and dh
    are formed: 13 E32.  (Its argument is exact: the largest logit is 0 and the scale 1.)"""
    k, cols = 16, 64
    table = torch.eye(cols, device=DEV)
    h = torch.full((50, cols), -200.0, device=DEV)
    h[:, 63] = 0.0
    ids = torch.arange(k, device=DEV).expand(50, k).contiguous()
    logits = -40 - 45 * torch.rand(50, k, device=DEV)
    logits[:, 0] = 0.0
    loss, lse = torch.empty(50, device=DEV), torch.empty(50, device=DEV)
    sizes = (50, cols, cols, k, F32)
    work = torch.empty(max(R.umap_rows_distill_workspace(*sizes), R.umap_rows_distill_grad_workspace(*sizes)), dtype=torch.uint8, device=DEV)
    dh = torch.empty_like(h)
    R.umap_rows_distill(h, table, ids, logits, loss, lse, work)
    R.umap_rows_distill_grad(h, table, ids, logits, lse, work, dh=dh)
    q = torch.softmax(logits.to(F64), 1)
    near(dh[:, :k], -q, 13 * E32 * q, "q")
