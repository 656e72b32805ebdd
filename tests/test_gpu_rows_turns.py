"""Norm and gradient with more rows than the workgroups of a launch take at once, so that each takes
several turns (reading ahead, exchanging sums in alternate buffers, adding to dweight): every way
in which rows lie in workgroups, every type, in place and not.  The references are formed on the
GPU in 64 bits."""

import pytest
import torch

import rows_reference as ref
from paper_2008_00325_amd import umap_rows as R
from test_gpu_rows import BF16, DEV, F16, F32, I8, Workspace, rand

pytestmark = pytest.mark.gpu
F64 = torch.float64

# columns: a thread a row; 8, 16, 32 or 64 lanes of one vector; of two; workgroups of one vector per thread, of two, of four.
# Rows: with dweight a workgroup takes 256, 32, 16, 8, 4, 4 rows, then one, and 1,280 workgroups at most run at once;
# without, or in the norm, 1,024 workgroups at least take four turns (two beyond 512 columns).
TURNS = {5: (600_000, 1_100_000), 64: (70_000, 140_000), 128: (20_000, 70_000), 256: (10_000, 35_000), 512: (10_000, 17_000),
         1000: (5000, 8300), 1040: (3000, 2100), 8192: (600, 2100), 9001: (600, 2100), 20001: (600, 600)}


def near(got, want, bound):
    off = (got.to(F64) - want).abs()
    bad = ~(off <= bound)
    rows = torch.nonzero(bad.reshape(bad.shape[0], -1).any(1))[:, 0]
    assert not rows.numel(), f"{rows.numel()} of {bad.shape[0]} rows off, the first {rows[:5].tolist()}"


def check(dy, h, w, dh, dx, want_dw):
    """dx may be dy or dh: the reference is formed first."""
    n, dim = dy.shape
    dx64, size, dw64, dw_size = ref.norm_grad(dy.to(F64), h.to(F64), w.to(F64), 1e-6, None if dh is None else dh.to(F64))
    dw = torch.full((dim,), 7.0, device=DEV) if want_dw else None
    work = Workspace(R.umap_rows_norm_grad_workspace(n, dim)) if want_dw else None
    R.umap_rows_norm_grad(dy, h, dx, weight=w, dh=dh, dweight=dw, workspace=work and work.inside)
    assert work is None or work.framed()
    steps = (-(-dim // 64) + 40) * ref.E32
    near(dx, dx64, ref.U[dy.dtype] * dx64.abs() + steps * size + ref.TINY[dy.dtype])
    if want_dw:
        # a workgroup's turns (8 at most), its lanes and waves, a stretch of the 1,280 sums, 16 stretches
        near(dw[:, None], dw64[:, None], (128 * ref.E32 + steps) * dw_size[:, None])


@pytest.mark.parametrize("dim", TURNS)
@pytest.mark.parametrize("want_dw", [True, False])
def test_norm_grad_in_several_turns(dim, want_dw):
    torch.manual_seed(dim)
    n = TURNS[dim][0 if want_dw else 1]
    for dtype, with_dh in ((F32, True), (F32, False), (F16, True), (BF16, False), (BF16, True)):
        dy, h = rand(n, dim, dtype), rand(n, dim, dtype, spread=2.0)
        w = (1 + 0.2 * torch.randn(dim, device=DEV)).to(dtype)
        check(dy, h, w, rand(n, dim, dtype) if with_dh else None, torch.empty_like(dy), want_dw)


@pytest.mark.parametrize("dim", TURNS)
@pytest.mark.parametrize("want_dw", [True, False])
def test_norm_grad_in_place_in_several_turns(dim, want_dw):
    torch.manual_seed(dim + 1)
    n = TURNS[dim][0 if want_dw else 1]
    for dtype, which in ((BF16, "dy"), (F32, "dh"), (F16, "dh")):
        dy, h, dh = rand(n, dim, dtype), rand(n, dim, dtype), rand(n, dim, dtype)
        check(dy, h, rand(1, dim, dtype)[0], dh, dy if which == "dy" else dh, want_dw)


@pytest.mark.parametrize("dim", TURNS)
def test_norm_in_several_turns(dim):
    torch.manual_seed(dim + 2)
    n = TURNS[dim][1]
    for dtype, residual, alias in ((F32, True, "residual"), (BF16, True, "x"), (F16, False, "x"), (F16, True, None)):
        x, r = rand(n, dim, dtype), rand(n, dim, dtype) if residual else None
        w = rand(1, dim, dtype)[0]
        x64, r64 = x.to(F64), None if r is None else r.to(F64)
        h64, y64 = ref.norm(x64, r64, w.to(F64), 1e-6)
        bound = ref.norm_bound(x64, r64, w.to(F64), 1e-6, dtype)
        off = ref.norm_bound(x64, r64, w.to(F64), 1e-6, F32)
        q, scales = torch.empty(n, dim, device=DEV, dtype=I8), torch.empty(n, 1, device=DEV)
        R.umap_rows_norm(x, q, weight=w, residual=r, y_scales=scales)
        near(q.to(F64) * scales.to(F64), y64, 0.5 * (1 + 1e-3) * scales.to(F64) + off + 4 * ref.E32 * y64.abs())
        h = r if alias == "residual" else x if alias == "x" else torch.empty_like(x)
        y = torch.empty_like(x)
        R.umap_rows_norm(x, y, weight=w, residual=r, h=h)
        near(y, y64, bound)
        parts = x64.abs() + (0 if r64 is None else r64.abs())
        near(h, h64, ref.U[dtype] * h64.abs() + 2 * ref.E32 * parts + ref.TINY[dtype])
