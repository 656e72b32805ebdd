"""Tensors that the row operators write are changed in place for autograd too."""

import pytest
import torch

from paper_2008_00325_amd import umap_rows as R
from test_gpu_rows import BF16, DEV, F32, I8

pytestmark = pytest.mark.gpu


def ones(*shape, t=F32):
    return torch.ones(*shape, device=DEV, dtype=t)


def writes():
    """Each call, and the tensors that it writes, by name."""
    ids = torch.tensor([1, 0, 2], device=DEV)
    out, grad = ones(3, 8), ones(5, 8)
    yield "lookup", lambda: R.umap_rows_lookup(ones(5, 8), ids, out), [out]
    for accumulate in (False, True):
        work = torch.empty(R.umap_rows_lookup_grad_workspace(3, 5, 8), dtype=torch.uint8, device=DEV)
        yield "grad", lambda: R.umap_rows_lookup_grad(ones(3, 8), ids, grad, work, accumulate=accumulate), [grad]
    y, q, scales, h = ones(3, 8), ones(3, 8, t=I8), ones(3), ones(3, 8)
    yield "norm", lambda: R.umap_rows_norm(ones(3, 8), y), [y]
    yield "norm in 8 bits", lambda: R.umap_rows_norm(ones(3, 8), q, y_scales=scales, h=h), [q, scales, h]
    dx, dw = ones(3, 8), ones(8)
    yield "norm grad", lambda: R.umap_rows_norm_grad(ones(3, 8), ones(3, 8), dx), [dx]
    work2 = torch.empty(R.umap_rows_norm_grad_workspace(3, 8), dtype=torch.uint8, device=DEV)
    yield "both", lambda: R.umap_rows_norm_grad(ones(3, 8), ones(3, 8), dx, dweight=dw, workspace=work2), [dx, dw]


def test_what_is_written_has_a_new_version():
    for name, call, written in writes():
        before = [x._version for x in written]
        call()
        assert all(x._version > v for x, v in zip(written, before)), name


def test_a_backward_pass_does_not_take_overwritten_values():
    table = torch.nn.Parameter(ones(5, 8))
    loss = (table * table).sum()   # keeps the table for its backward pass
    work = torch.empty(R.umap_rows_lookup_grad_workspace(3, 5, 8), dtype=torch.uint8, device=DEV)
    R.umap_rows_lookup_grad(ones(3, 8), torch.tensor([1, 0, 2], device=DEV), table, work, scale=-0.1, accumulate=True)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_under_inference_mode():
    with torch.inference_mode():
        out = torch.empty(2, 8, device=DEV, dtype=BF16)
        R.umap_rows_lookup(ones(5, 8), torch.tensor([4, 0], device=DEV), out)
        assert bool((out == 1).all())
