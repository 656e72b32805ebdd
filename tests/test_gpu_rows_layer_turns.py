"""Sums of the layer norm's gradient where workgroups take several turns of rows: with whole numbers, whose sums are exact in any
order, so that a row left out or counted twice shows."""

import pytest
import torch

from paper_2008_00325_amd import umap_rows as R
from rows_reference import E32
from test_gpu_rows import BF16, DEV, F32, FLOATS, Workspace
from test_gpu_rows_head import F64, near
from test_gpu_rows_layer import Norm

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seed():
    torch.manual_seed(31)
    yield
    torch.cuda.synchronize()


def grads(dy, h, dx=None, eps=0.0):
    n, cols = h.shape
    dw, db = torch.full((cols,), 7.0, device=DEV), torch.full((cols,), 7.0, device=DEV)
    dx = torch.empty_like(h) if dx is None else dx
    work = Workspace(R.umap_rows_layer_norm_grad_workspace(n, cols))
    R.umap_rows_layer_norm_grad(dy, h, dx, dweight=dw, dbias=db, workspace=work.inside, eps=eps)
    assert work.framed()
    return dx, dw, db


def whole(n, cols, dtype):
    """Numbers of 1 to 3 with either sign."""
    return (torch.randint(1, 4, (n, cols), device=DEV) * (torch.randint(0, 2, (n, cols), device=DEV) * 2 - 1)).to(dtype)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("n,cols", [(130_001, 4), (70_001, 16), (70_001, 64), (40_001, 128), (20_001, 256), (12_001, 512), (9001, 1024),
                                    (5001, 2048), (3001, 4096), (2001, 8192), (1301, 16384), (1301, 32768)])
def test_rows_of_plus_and_minus_one(n, cols, dtype):
    """Half of a row is 1, half -1: mean 0, variance 1, so with eps = 0 u = h, and every sum is a whole number below 2^24 (a power of
    two of columns: the mean is exact)."""
    h = torch.ones(n, cols, device=DEV)
    h[:, :cols // 2] = -1
    h = torch.where(torch.rand(n, 1, device=DEV) < 0.5, h, -h)
    turned = [torch.roll(h, int(by), 1) for by in torch.randint(0, cols, (3,))]   # other orders
    which = torch.randint(0, 3, (n, 1), device=DEV)
    h = torch.where(which == 0, turned[0], torch.where(which == 1, turned[1], turned[2])).to(dtype)
    dy = whole(n, cols, dtype)
    _, dw, db = grads(dy, h)
    assert torch.equal(db.to(F64), dy.to(F64).sum(0))
    assert torch.equal(dw.to(F64), (dy.to(F64) * h.to(F64)).sum(0))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,cols", [(130_001, 5), (70_001, 24), (40_001, 100), (20_001, 200), (12_001, 300), (9001, 1001), (3001, 5000),
                                    (1301, 20_003)])
def test_odd_columns(n, cols, dtype):
    """dbias is exact; dweight's terms go through at most 100 additions each: the turns of a workgroup, its lanes and waves, 16
    stretches of the workgroups and those."""
    h, dy = torch.randn(n, cols, device=DEV).to(dtype), whole(n, cols, dtype)
    dx, dw, db = grads(dy, h, eps=1e-5)
    assert torch.equal(db.to(F64), dy.to(F64).sum(0))
    norm = Norm(h.to(F64), None, 1e-5)
    t = dy.to(F64) * norm.u
    near(dw, t.sum(0), (dy.to(F64).abs() * norm.u_err).sum(0) + 100 * E32 * t.abs().sum(0), "dweight")
    want, bound = norm.grad(dy.to(F64), torch.tensor(1.0, dtype=F64, device=DEV), None, dtype)[:2]
    near(dx, want, bound, "dx")
    # in place of dy, whose sums are the same
    again = grads(dy, h, dx=dy, eps=1e-5)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dw) and torch.equal(again[2], db)
