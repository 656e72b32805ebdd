"""Boundary of the layer norm's calls that needs no GPU: what is refused before any HIP call."""

import pytest
import torch

from paper_2008_00325_amd import umap_layout as U
from paper_2008_00325_amd import umap_rows as R
from test_rows_binding import On, two_gpus  # noqa: F401
from test_rows_boundary import A, refused, rows


def test_layer_norm_refuses():
    ok = dict(x=rows(A), r=rows(2 * A), h=rows(3 * A), w=4 * A, wt=R.UMAP_F32, b=6 * A, bt=R.UMAP_BF16, e=1e-5, y=rows(5 * A))

    def f(**kw):
        v = {**ok, **kw}
        return R.lib().umap_rows_layer_norm(v["x"], v["r"], v["h"], v["w"], v["wt"], v["b"], v["bt"], v["e"], v["y"], None)

    refused(f(x=None), "x must not be NULL")
    refused(f(y=None), "y must not be NULL")
    refused(f(x=rows(A, type=R.UMAP_I8, scales=7 * A)), "element type")
    refused(f(y=rows(5 * A, type=R.UMAP_I8, scales=7 * A)), "element type")
    refused(f(x=rows(A, cols=32769), y=rows(5 * A, cols=32769)), "cols")
    refused(f(x=rows(A, n=2**31), y=rows(5 * A, n=2**31)), "rows must be")
    refused(f(y=rows(5 * A, cols=17)), "cols")
    refused(f(y=rows(5 * A, n=11)), "y has 11 rows")
    refused(f(r=rows(2 * A, n=9)), "residual has 9 rows")
    refused(f(r=rows(2 * A, type=R.UMAP_BF16)), "residual must have x's type")
    refused(f(h=rows(3 * A, type=R.UMAP_F16)), "h must have x's type")
    refused(f(h=rows(3 * A, n=11)), "h has 11 rows")
    refused(f(w=4 * A + 2), "weight is not aligned")
    refused(f(b=6 * A + 1), "bias is not aligned")
    refused(f(wt=R.UMAP_I8), "weight_type")
    refused(f(bt=7), "bias_type")
    refused(f(e=-1e-6), "eps")
    refused(f(e=float("inf")), "eps")
    for at in (A, 2 * A, 3 * A, 4 * A, 6 * A):
        refused(f(y=rows(at)), "y overlaps")
    refused(f(h=rows(A + 64)), "h overlaps")
    refused(f(h=rows(A, stride=17)), "h overlaps")
    for at in (4 * A, 6 * A):
        refused(f(h=rows(at)), "h overlaps")
    assert f(x=rows(0, n=0), y=rows(0, n=0), r=None, h=None) == U.UMAP_OK


def test_layer_norm_grad_refuses():
    L = R.lib()
    need = L.umap_rows_layer_norm_grad_workspace(10, 16)
    assert need > 0
    ok = dict(dy=rows(A), h=rows(2 * A), dh=rows(3 * A), w=4 * A, wt=R.UMAP_F32, e=1e-6, dx=rows(5 * A), dw=6 * A, db=8 * A,
              ws=7 * A, wb=need)

    def f(**kw):
        v = {**ok, **kw}
        return L.umap_rows_layer_norm_grad(v["dy"], v["h"], v["dh"], v["w"], v["wt"], v["e"], v["dx"], v["dw"], v["db"], v["ws"], v["wb"], None)

    for name in ("dy", "h", "dx"):
        refused(f(**{name: None}), f"{name} must not be NULL")
    refused(f(h=rows(2 * A, n=9)), "h has 9 rows")
    refused(f(dx=rows(5 * A, cols=15)), "dx has 15 cols")
    refused(f(dh=rows(3 * A, type=R.UMAP_BF16)), "one type")
    refused(f(dy=rows(A, n=2**31)), "rows must be")
    refused(f(e=float("inf")), "eps")
    refused(f(wt=9), "weight_type")
    refused(f(dw=6 * A + 1), "dweight is not aligned")
    refused(f(db=8 * A + 2), "dbias is not aligned")
    for only in (dict(), dict(dw=None), dict(db=None)):
        refused(f(ws=None, **only), "workspace of 0 bytes")
        refused(f(wb=need - 1, **only), "workspace of")
        refused(f(ws=7 * A + 4, **only), "aligned to 16")
    for at in (2 * A, A + 64, 3 * A + 64, 4 * A, 6 * A, 8 * A, 7 * A):
        refused(f(dx=rows(at)), "dx overlaps")
    for at in (A, 2 * A, 3 * A, 4 * A, 8 * A, 7 * A):
        refused(f(dw=at), "dweight overlaps")
    for at in (A, 2 * A, 3 * A, 4 * A, 7 * A):
        refused(f(db=at), "dbias overlaps")
    refused(f(ws=2 * A), "workspace overlaps")
    for bad in ((-1, 16), (2**31, 16), (10, 0), (10, 32769)):
        assert L.umap_rows_layer_norm_grad_workspace(*bad) == U.UMAP_E_INVAL
    assert f(dy=rows(0, n=0), h=rows(0, n=0), dh=None, dx=rows(0, n=0), dw=None, db=None) == U.UMAP_OK


def calls():
    f32, u8 = torch.float32, torch.uint8
    yield R.umap_rows_layer_norm, dict(x=(4, 8, f32), y=(4, 8, f32), weight=(8, f32), bias=(8, f32), residual=(4, 8, f32), h=(4, 8, f32))
    yield R.umap_rows_layer_norm_grad, dict(dy=(4, 8, f32), h=(4, 8, f32), dx=(4, 8, f32), weight=(8, f32), dh=(4, 8, f32),
                                            dweight=(8, f32), dbias=(8, f32), workspace=(9999, u8))


@pytest.mark.parametrize("call,tensors", calls(), ids=lambda x: getattr(x, "__name__", ""))
def test_tensors_that_do_not_fit_are_refused(two_gpus, monkeypatch, call, tensors):  # noqa: F811
    def no_call(*args):
        raise AssertionError("the library was called")

    R.lib()
    monkeypatch.setitem(R._call, call.__name__, no_call)

    def given(other=None, at=1, shorter=None):
        return {name: On(at if name == other else 0, *((t[0] - (name == shorter),) + t[1:-1]), dtype=t[-1]) for name, t in tensors.items()}

    with pytest.raises(AssertionError, match="the library was called"):
        call(**given())
    for name in tensors:
        with pytest.raises(ValueError, match="lies on GPU 1, the current one is 0"):
            call(**given(name))
        with pytest.raises(ValueError, match="must be a GPU tensor"):
            call(**given(name, -1))
    for name in set(tensors) & {"weight", "bias", "dweight", "dbias"}:
        with pytest.raises(ValueError, match="columns|the call needs"):
            call(**given(shorter=name))
