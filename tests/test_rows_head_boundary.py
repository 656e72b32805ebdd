"""Boundary of the head's calls that needs no GPU: every invalid argument is refused before any HIP call,
by the library or by the binding, and the stated limits are the enforced ones."""

import os
import re

import pytest
import torch

from paper_2008_00325_amd import umap_layout as U
from paper_2008_00325_amd import umap_rows as R
from test_rows_binding import On, two_gpus  # noqa: F401
from test_rows_boundary import A, refused, rows

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "umap_rows.h")
BF = R.UMAP_BF16
N, V, C, K = 10, 30, 16, 4   # rows, tokens, columns, a teacher's tokens


def loss_call(taught, **kw):
    need = R.lib().umap_rows_distill_workspace(N, V, C, K, BF)
    v = dict(h=rows(A, N, C, BF), w=rows(2 * A, V, C, BF), i=3 * A, it=R.UMAP_I64, t=rows(4 * A, N, K), s=1.0, ts=1.0, loss=5 * A,
             lse=6 * A, ws=7 * A, wb=need) | kw
    if taught:
        return R.lib().umap_rows_distill(v["h"], v["w"], v["i"], v["it"], v["t"], v["s"], v["ts"], v["loss"], v["lse"], v["ws"], v["wb"], None)
    return R.lib().umap_rows_cross_entropy(v["h"], v["w"], v["i"], v["it"], v["s"], v["loss"], v["lse"], v["ws"], v["wb"], None)


def grad_call(taught, **kw):
    need = R.lib().umap_rows_distill_grad_workspace(N, V, C, K, BF)
    v = dict(h=rows(A, N, C, BF), w=rows(2 * A, V, C, BF), i=3 * A, it=R.UMAP_I64, t=rows(4 * A, N, K), s=1.0, ts=1.0, lse=6 * A,
             dl=8 * A, ds=1.0, dh=rows(9 * A, N, C, BF), dw=rows(10 * A, V, C, BF), a=0, ws=7 * A, wb=need) | kw
    if taught:
        return R.lib().umap_rows_distill_grad(v["h"], v["w"], v["i"], v["it"], v["t"], v["s"], v["ts"], v["lse"], v["dl"], v["ds"],
                                              v["dh"], v["dw"], v["a"], v["ws"], v["wb"], None)
    return R.lib().umap_rows_cross_entropy_grad(v["h"], v["w"], v["i"], v["it"], v["s"], v["lse"], v["dl"], v["ds"], v["dh"],
                                                v["dw"], v["a"], v["ws"], v["wb"], None)


@pytest.mark.parametrize("taught", [False, True])
@pytest.mark.parametrize("call", [loss_call, grad_call])
def test_both_refuse(call, taught):
    def f(**kw):
        return call(taught, **kw)

    refused(f(h=None), "h must not be NULL")
    refused(f(w=None), "table must not be NULL")
    refused(f(i=None), "must not be NULL")
    refused(f(h=rows(A, N, C, R.UMAP_I8, scales=11 * A)), "element type")
    refused(f(w=rows(2 * A, V, C, R.UMAP_F8, scales=11 * A)), "element type")
    refused(f(w=rows(2 * A, V, C, R.UMAP_F16)), "table must have h's type")
    refused(f(w=rows(2 * A, V, C + 1, BF)), "cols")
    refused(f(w=rows(2 * A, 0, C, BF)), "rows of table")
    refused(f(w=rows(2 * A, 1 << 26, C, BF)), "rows of table")
    refused(f(h=rows(A, 1 << 24, C, BF), t=rows(4 * A, 1 << 24, K)), "rows of h")
    refused(f(h=rows(A, N, 32769, BF), w=rows(2 * A, V, 32769, BF)), "cols")
    refused(f(h=rows(A, N, C, BF, stride=C - 1)), "stride")
    refused(f(it=R.UMAP_F32), "id_type")
    refused(f(i=3 * A + 4), "ids are not aligned")
    refused(f(s=float("nan")), "scale")
    refused(f(s=float("inf")), "scale")
    refused(f(lse=None), "lse must not be NULL")
    refused(f(lse=6 * A + 2), "lse is not aligned")
    refused(f(ws=None), "workspace of 0 bytes")
    refused(f(wb=15), "workspace of 15 bytes")
    refused(f(ws=7 * A + 8), "aligned to 16")
    refused(f(ws=A), "workspace overlaps")
    refused(f(ws=2 * A - 16), "workspace overlaps")
    refused(f(ws=3 * A), "workspace overlaps")
    refused(f(ws=6 * A - 16), "overlaps")
    if taught:
        refused(f(t=None), "teacher must not be NULL")
        refused(f(t=rows(4 * A, N + 1, K)), "teacher has 11 rows")
        refused(f(t=rows(4 * A, N, 257)), "cols")
        refused(f(t=rows(4 * A, N, K, R.UMAP_I8, scales=11 * A)), "element type")
        refused(f(ts=float("nan")), "teacher_scale")
        refused(f(ws=4 * A), "workspace overlaps")


@pytest.mark.parametrize("taught", [False, True])
def test_loss_refuses(taught):
    refused(loss_call(taught, loss=None), "loss must not be NULL")
    refused(loss_call(taught, loss=5 * A + 1), "loss is not aligned")
    for at in (A, 2 * A + 4, 3 * A + 4, 6 * A + 36, 7 * A):
        refused(loss_call(taught, loss=at), "loss overlaps")
    for at in (A, 2 * A + 4, 3 * A + 4, 7 * A):
        refused(loss_call(taught, lse=at), "lse overlaps")
    none = rows(0, 0, C, BF)
    assert loss_call(taught, h=none, i=None, t=rows(0, 0, K), loss=None, lse=None) == U.UMAP_OK


@pytest.mark.parametrize("taught", [False, True])
def test_grad_refuses(taught):
    def f(**kw):
        return grad_call(taught, **kw)

    refused(f(dh=None, dw=None), "must not both be NULL")
    refused(f(dl=8 * A + 1), "dloss is not aligned")
    refused(f(ds=float("inf")), "dscale")
    refused(f(a=2), "accumulate")
    refused(f(dh=rows(9 * A, N + 1, C, BF)), "dh has 11 rows")
    refused(f(dh=rows(9 * A, N, C + 1, BF)), "dh has 17 cols")
    refused(f(dh=rows(9 * A, N, C)), "dh must have h's type")
    refused(f(dw=rows(10 * A, V - 1, C, BF)), "dtable has 29 rows")
    refused(f(dw=rows(10 * A, V, C)), "dtable must have table's type")
    refused(f(dh=rows(9 * A, N, C, BF, stride=0)), "stride")
    for at in (A, 2 * A, 3 * A, 6 * A, 8 * A, 10 * A, 7 * A):
        refused(f(dh=rows(at, N, C, BF)), "dh overlaps")
    for at in (A, 2 * A + 32, 3 * A, 6 * A, 8 * A, 7 * A):
        refused(f(dw=rows(at, V, C, BF)), "dtable overlaps")
    refused(f(ws=8 * A), "workspace overlaps")
    none = dict(h=rows(0, 0, C, BF), i=None, t=rows(0, 0, K), lse=None, dl=None, dh=rows(0, 0, C, BF))
    assert f(**none, dw=None) == U.UMAP_OK
    assert f(**none, a=1) == U.UMAP_OK


def test_workspaces_refuse_what_the_calls_refuse():
    L = R.lib()
    for f in (L.umap_rows_cross_entropy_workspace, L.umap_rows_cross_entropy_grad_workspace):
        assert f(0, 1, 1, BF) > 0 and f((1 << 24) - 1, (1 << 26) - 1, 32768, R.UMAP_F32) > 0
        for bad in ((-1, 1, 1, BF), (1 << 24, 1, 1, BF), (1, 0, 1, BF), (1, 1 << 26, 1, BF), (1, 1, 0, BF), (1, 1, 32769, BF), (1, 1, 1, R.UMAP_I8)):
            assert f(*bad) == U.UMAP_E_INVAL
    for f in (L.umap_rows_distill_workspace, L.umap_rows_distill_grad_workspace):
        assert f(0, 1, 1, 256, BF) > 0
        for k in (0, 257):
            assert f(1, 1, 1, k, BF) == U.UMAP_E_INVAL


def test_limits_are_stated():
    text = open(HEADER).read()
    comment = next(c for c in re.findall(r"/\*(.*?)\*/", text, flags=re.S) if "umap_rows_cross_entropy --" in c)
    assert "cols 1 .. 32768, rows < 2^24" in comment and "1 <= rows < 2^26" in comment
    assert "1 <= k <= 256" in text


def test_binding_refuses():
    cpu = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="GPU tensor"):
        R.umap_rows_cross_entropy(cpu, cpu, cpu, cpu, cpu, cpu)
    with pytest.raises(ValueError, match="must not hold"):
        R.umap_rows_distill(cpu.double(), cpu, cpu, cpu, cpu, cpu, cpu)
    with pytest.raises(ValueError, match="rows must not hold"):
        R.umap_rows_cross_entropy_workspace(4, 4, 4, torch.int8)
    with pytest.raises(U.UmapLayoutError, match="rows of table"):
        R.umap_rows_distill_grad_workspace(4, 0, 4, 4, torch.float32)


def calls():
    f32, i64, u8 = torch.float32, torch.int64, torch.uint8
    base = dict(h=(4, 8, f32), table=(9, 8, f32))
    tail = dict(lse=(4, f32), workspace=(99999, u8))
    grads = dict(dh=(4, 8, f32), dtable=(9, 8, f32), dloss=(4, f32))
    teach = dict(ids=(8, i64), teacher=(4, 2, f32))
    yield R.umap_rows_cross_entropy, base | dict(targets=(4, i64), loss=(4, f32)) | tail
    yield R.umap_rows_cross_entropy_grad, base | dict(targets=(4, i64)) | tail | grads
    yield R.umap_rows_distill, base | teach | dict(loss=(4, f32)) | tail
    yield R.umap_rows_distill_grad, base | teach | tail | grads


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
    for name in set(tensors) & {"targets", "ids", "loss", "lse", "dloss"}:
        with pytest.raises(ValueError, match="the call needs"):
            call(**given(shorter=name))
