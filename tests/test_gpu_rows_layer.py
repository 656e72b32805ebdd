"""Mean and variance norm of rows and its gradient on the GPU against their definitions in 64 bits, at the
sizes, strides and values where they can go wrong.  Bounds: fp32 sums of n terms are off by at most (n / threads of a
row + 24) E32 times the sum of the terms' magnitudes, with one rounding per output (rows_reference)."""

import math

import pytest
import torch

from paper_2008_00325_amd import umap_rows as R
from rows_reference import E32, TINY, U
from test_gpu_rows import BF16, DEV, F16, F32, FLOATS, Workspace, frame_untouched, hole, rand
from test_gpu_rows_head import near

pytestmark = pytest.mark.gpu
F64 = torch.float64
DIMS = [1, 2, 3, 7, 8, 9, 31, 63, 64, 65, 100, 127, 128, 200, 256, 257, 300, 512, 513, 784, 1001, 1024, 1025, 2056, 4100, 8192, 8193,
        9001, 16384]
WIDE = [16385, 20_003, 32768]


@pytest.fixture(autouse=True)
def _seed():
    torch.manual_seed(7)
    yield
    torch.cuda.synchronize()


def steps_of(cols):
    """Terms that one lane adds in turn (a row has 8 lanes up to 64 columns, 16 up to 128, .. 64 from 257 on), and the tree."""
    lanes = 8 if cols <= 64 else 16 if cols <= 128 else 32 if cols <= 256 else 64
    return -(-cols // lanes) + 24


class Norm:
    """h64: the exact rows, parts64: the magnitudes of what they are the sum of (or None: they are given)."""

    def __init__(self, h64, parts64, eps):
        self.cols = h64.shape[1]
        self.steps = steps_of(self.cols) * E32
        mean = h64.mean(1, keepdim=True)
        self.off = h64 - mean
        size = h64.abs().mean(1, keepdim=True)
        # h's own rounding; the mean's is corrected, up to what rounding leaves of the differences and of their mean
        own = torch.zeros_like(h64) if parts64 is None else E32 * parts64
        away = self.off.abs() + self.steps * size
        self.off_err = own + own.mean(1, keepdim=True) + 2 * E32 * away + self.steps * away.mean(1, keepdim=True)
        # fp32's values are multiples of 2^-149: the mean, and the mean of what it left, are off by up to 2^-150 each where
        # they lie among the smallest.  With a vanishing eps the differences are scaled up before the second mean, which
        # then takes the first one's error off again
        self.off_err = self.off_err + (2.0**-149 if eps >= 2.0**-62 else 0.0)
        var = (self.off * self.off).mean(1, keepdim=True)
        self.rho = 1 / torch.sqrt(var + eps)
        var_err = (2 * self.off.abs() * self.off_err + self.off_err**2 + self.steps * away**2).mean(1, keepdim=True)
        self.rho_err = self.rho * (torch.clamp(0.5 * var_err * self.rho**2, max=0.5) * 1.5 + 4 * E32)
        self.u = self.off * self.rho
        self.u_err = self.off_err * self.rho + (self.off.abs() + self.off_err) * self.rho_err + 2 * E32 * self.u.abs()

    def y(self, w64, b64, dtype):
        y = self.u * w64 + b64
        err = self.u_err * w64.abs() + 2 * E32 * (y.abs() + (self.u * w64).abs())
        return y, err + U[dtype] * (y.abs() + err) + TINY[dtype]

    def grad(self, dy64, w64, dh64, dtype):
        g = dy64 * w64
        n, cols = dy64.shape
        mean_g, along = g.mean(1, keepdim=True), (g * self.u).mean(1, keepdim=True)
        dx = self.rho * (g - mean_g - self.u * along)
        ga = g.abs()
        mean_err = (self.steps + 3 * E32) * ga.mean(1, keepdim=True)
        along_err = (ga * (self.u_err + (self.steps + 3 * E32) * self.u.abs())).mean(1, keepdim=True)
        inner = ga + mean_g.abs() + (self.u * along).abs()
        err = self.rho * (mean_err + self.u_err * along.abs() + self.u.abs() * along_err + 4 * E32 * inner) + self.rho_err * inner
        if dh64 is not None:
            dx = dx + dh64
            err = err + E32 * (dx.abs() + dh64.abs())
        t = dy64 * self.u
        # rows of a workgroup one after the other, then the workgroups
        sums = (n + 64) * E32
        dw_err = (dy64.abs() * self.u_err).sum(0) + sums * t.abs().sum(0)
        return (dx, err + U[dtype] * (dx.abs() + err) + TINY[dtype], t.sum(0), dw_err + 1e-37, dy64.sum(0),
                sums * dy64.abs().sum(0) + 1e-37)


def vector(cols, dtype, mean):
    return None if dtype is None else (mean + 0.3 * torch.randn(cols, device=DEV)).to(dtype)


def as64(x, other):
    return torch.tensor(other, dtype=F64, device=DEV) if x is None else x.to(F64)


def check_norm(n, cols, x_type, y_type, residual=False, keep=None, w=F32, b=F32, pad=0, shift=0, eps=1e-5, x=None):
    if x is None:
        x = rand(n, cols, x_type, pad, shift, 2.0)
        x += 0.7
    r = rand(n, cols, x_type, shift, pad) if residual else None
    W, B = vector(cols, w, 1.0), vector(cols, b, 0.0)
    h64 = x.to(F64) + (r.to(F64) if residual else 0)
    parts = h64.abs() if residual else None
    whole, y = hole(n, cols, y_type, pad, shift)
    whole_h, h = hole(n, cols, x_type, shift, pad)
    if keep in ("x", "residual"):
        h, whole_h = (x.clone() if keep == "x" else r.clone()), None
    args = dict(x=h if keep == "x" else x, residual=h if keep == "residual" else r)
    R.umap_rows_layer_norm(args["x"], y, weight=W, bias=B, residual=args["residual"], h=h if keep else None, eps=eps)
    want, bound = Norm(h64, parts, eps).y(as64(W, 1.0), as64(B, 0.0), y_type)
    near(y, want, bound, "y")
    assert frame_untouched(whole, cols, shift)
    if keep:
        near(h, h64, (U[x_type] + 2 * E32) * h64.abs() + TINY[x_type], "h")
        assert whole_h is None or frame_untouched(whole_h, cols, pad)


def check_grad(n, cols, dtype, upstream=False, w=F32, pad=0, shift=0, eps=1e-5, into=None, h=None, sums="both"):
    h = rand(n, cols, dtype, pad, shift, 2.0) + 0.5 if h is None else h
    dy = rand(n, cols, dtype, shift, pad)
    dh = rand(n, cols, dtype) if upstream else None
    W = vector(cols, w, 1.0)
    want = Norm(h.to(F64), None, eps).grad(dy.to(F64), as64(W, 1.0), None if dh is None else dh.to(F64), dtype)
    whole, dx = hole(n, cols, dtype, pad, shift)
    if into == "dy":
        dx, whole = dy, None
    elif into == "dh":
        dx, whole = dh, None
    frames = [torch.full((cols + 1,), 7.0, device=DEV) for _ in range(2)]
    dw, db = frames[0][:cols], frames[1][:cols]
    work = Workspace(R.umap_rows_layer_norm_grad_workspace(n, cols))
    R.umap_rows_layer_norm_grad(dy, h, dx, weight=W, dh=dh, dweight=dw if sums in ("both", "weight") else None,
                                dbias=db if sums in ("both", "bias") else None, workspace=work.inside if sums else None, eps=eps)
    near(dx, want[0], want[1], "dx")
    for name, got, at in (("weight", dw, 2), ("bias", db, 4)):
        if sums in ("both", name):
            near(got, want[at], want[at + 1], name)
        else:
            assert bool((got == 7).all())
    assert all(float(f[cols]) == 7 for f in frames) and work.framed()
    assert whole is None or frame_untouched(whole, cols, shift)


@pytest.mark.parametrize("cols", DIMS + WIDE)
@pytest.mark.parametrize("x_type,y_type", [(F32, F32), (BF16, BF16), (F16, F32), (F32, BF16), (BF16, F16)])
def test_norm_dims(cols, x_type, y_type):
    check_norm(37, cols, x_type, y_type)
    check_norm(5, cols, x_type, y_type, residual=True, keep="new", w=x_type, b=None)


@pytest.mark.parametrize("cols", DIMS + WIDE)
@pytest.mark.parametrize("dtype", FLOATS)
def test_grad_dims(cols, dtype):
    check_grad(37, cols, dtype)
    check_grad(5, cols, dtype, upstream=True, w=dtype)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("pad,shift", [(1, 0), (8, 0), (0, 1), (5, 3)])
def test_strides_and_alignment(dtype, pad, shift):
    for cols in (3, 64, 301, 1500):
        check_norm(70, cols, dtype, dtype, pad=pad, shift=shift, residual=True, keep="new", w=BF16, b=F16)
        check_grad(70, cols, dtype, pad=pad, shift=shift, w=None)


@pytest.mark.parametrize("n,cols", [(1, 1), (1, 9001), (9000, 16), (70_001, 5), (20_000, 300), (3000, 1024), (2100, 4096), (1400, 9001), (700, 17_000)])
def test_many_rows(n, cols):
    for dtype in (BF16, F32):
        check_norm(n, cols, dtype, dtype, residual=True, keep="new")
        check_grad(n, cols, dtype, upstream=True)


@pytest.mark.parametrize("cols", [6, 100, 700, 5000, 12_000, 20_000])
def test_in_place(cols):
    for keep in ("x", "residual"):
        check_norm(300, cols, BF16, BF16, residual=True, keep=keep)
    check_norm(300, cols, F32, F16, keep="x")
    for into in ("dy", "dh"):
        check_grad(300, cols, BF16, upstream=True, into=into)


@pytest.mark.parametrize("cols", [5, 300, 3000, 20_000])
@pytest.mark.parametrize("sums", ["weight", "bias", None])
def test_either_sum_alone(cols, sums):
    check_grad(120, cols, F16, sums=sums)


@pytest.mark.parametrize("cols", [2, 50, 700, 3000, 17_000])
def test_rows_whose_mean_is_far_from_zero(cols):
    x = 1000.0 + rand(60, cols, F32)
    check_norm(60, cols, F32, F32, x=x)
    check_grad(60, cols, F32, h=x)


@pytest.mark.parametrize("cols", [3, 50, 700, 3000, 17_000])
@pytest.mark.parametrize("size", [1e-42, 1e-30, 1e-20, 1e18, 1e30, 3e38 / 4])
def test_ends_of_the_range(cols, size):
    """Rows whose squares leave fp32's range, with and without a mean far from zero, eps 0 and not."""
    x = torch.randn(30, cols, device=DEV).clamp(-4, 4) * size
    if size < 1e-40:   # subnormal values have few digits: take what they are
        x = x.to(F32)
    for eps in (0.0, 1e-5):
        want, bound = Norm(x.to(F64), None, eps).y(as64(None, 1.0), as64(None, 0.0), F32)
        y = torch.empty_like(x)
        R.umap_rows_layer_norm(x, y, eps=eps)
        fine = (x.to(F64).var(1, correction=0) > 0) | (eps > 0)
        near(y[fine], want[fine], bound[fine])
        if size in (1e-30, 1e30):
            dy = torch.randn_like(x)
            dx, dw, db = torch.empty_like(x), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
            work = Workspace(R.umap_rows_layer_norm_grad_workspace(30, cols))
            R.umap_rows_layer_norm_grad(dy, x, dx, dweight=dw, dbias=db, workspace=work.inside, eps=eps)
            want = Norm(x.to(F64), None, eps).grad(dy.to(F64), as64(None, 1.0), None, F32)
            near(dx, want[0], want[1], "dx")
            near(dw, want[2], want[3], "dw")
            near(db, want[4], want[5], "db")


@pytest.mark.parametrize("value", [0.0, 1.1, 1234.567, 1e-30, -3e38, 1e-42])
def test_rows_of_equal_values(value):
    """Their differences are zeros, not their mean's rounding."""
    for cols in (1, 8, 100, 300, 4095, 20_000):
        x = torch.full((9, cols), value, device=DEV)
        y, b = torch.empty_like(x), torch.randn(cols, device=DEV)
        R.umap_rows_layer_norm(x, y, bias=b)
        assert torch.equal(y, b.expand_as(y)) if abs(value) > 1e-29 or value == 0 else bool(((y - b).abs() < 1e-20).all())
        R.umap_rows_layer_norm(x, y, eps=0.0)
        assert bool(y.isnan().all())
        # one value apart
        x[:, cols // 2] *= 1.0 + 2.0**-10
        for eps in (0.0, 1e-5):
            R.umap_rows_layer_norm(x, y, eps=eps)
            # 0 and the smallest values do not change by a factor, and one column has no spread: 0 / 0 as above
            if eps > 0 or float(x.to(F64).var(1, correction=0).min()) > 0:
                want, bound = Norm(x.to(F64), None, eps).y(as64(None, 1.0), as64(None, 0.0), F32)
                near(y, want, bound)


def test_rows_that_are_not_finite():
    for cols in (5, 40, 900, 3000, 17_000):
        x = rand(6, cols, F32)
        x[1, cols // 2] = math.nan
        x[2, 0] = math.inf
        x[3, cols - 1] = -math.inf
        y = torch.empty_like(x)
        R.umap_rows_layer_norm(x, y)
        assert bool(y[1:4].isnan().all()) and bool(torch.isfinite(y[[0, 4, 5]]).all())


def test_empty_calls():
    none = torch.empty(0, 24, device=DEV)
    R.umap_rows_layer_norm(none, none.clone())
    dw, db = torch.ones(24, device=DEV), torch.ones(24, device=DEV)
    work = Workspace(R.umap_rows_layer_norm_grad_workspace(0, 24))
    R.umap_rows_layer_norm_grad(none, none.clone(), none.clone(), dweight=dw, dbias=db, workspace=work.inside)
    assert not bool(dw.any()) and not bool(db.any())


@pytest.mark.parametrize("cols", [7, 300])
def test_gradient_against_differences(cols):
    h, dy = torch.randn(6, cols, device=DEV), torch.randn(6, cols, device=DEV)
    W, B = vector(cols, F32, 1.0), vector(cols, F32, 0.0)
    dx, dw, db = torch.empty_like(h), torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    work = Workspace(R.umap_rows_layer_norm_grad_workspace(6, cols))
    R.umap_rows_layer_norm_grad(dy, h, dx, weight=W, dweight=dw, dbias=db, workspace=work.inside)
    for x, g in ((h, dx), (W, dw), (B, db)):
        along, base, value = torch.randn_like(x), x.clone(), []
        for step in (1e-2, -1e-2):
            x.copy_(base + step * along)
            y = torch.empty_like(h)
            R.umap_rows_layer_norm(h, y, weight=W, bias=B)
            value.append(float((y.to(F64) * dy).sum()))
        x.copy_(base)
        slope = (value[0] - value[1]) / 2e-2
        # a third derivative times step^2 / 6, and 6 cols roundings of about 1e-7 over 2e-2
        assert abs(slope - float((g * along).sum())) < 1e-2 * (1 + abs(slope))


def test_same_bits_at_every_call_on_a_stream_and_new_versions():
    for cols in (300, 5000, 20_000):
        h, dy = rand(900, cols, BF16), rand(900, cols, BF16)
        outs = []
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for stream in (None, None, side):
            y, dx = torch.empty_like(h), torch.empty_like(h)
            dw, db = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
            work = torch.empty(R.umap_rows_layer_norm_grad_workspace(900, cols), dtype=torch.uint8, device=DEV)
            torch.cuda.synchronize()
            before = [x._version for x in (y, dx, dw, db)]
            R.umap_rows_layer_norm(h, y, stream=stream)
            R.umap_rows_layer_norm_grad(dy, h, dx, dweight=dw, dbias=db, workspace=work, stream=stream)
            torch.cuda.synchronize()
            assert all(x._version > v for x, v in zip((y, dx, dw, db), before))
            outs.append((y, dx, dw, db))
        assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(outs[0], o))


@pytest.mark.parametrize("cols", [100, 3000, 20_000])
def test_one_row_for_all(cols):
    """Inputs of stride 0 give the bits that their copies give."""
    n = 70
    one, other, more = (rand(1, cols, BF16).expand(n, cols) for _ in range(3))
    assert one.stride(0) == 0
    outs = []
    for x, dy, r in ((one, other, more), (one.contiguous(), other.contiguous(), more.contiguous())):
        y, h, dx = (torch.empty(n, cols, dtype=BF16, device=DEV) for _ in range(3))
        dw, db = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
        work = Workspace(R.umap_rows_layer_norm_grad_workspace(n, cols))
        R.umap_rows_layer_norm(x, y, residual=r, h=h)
        R.umap_rows_layer_norm_grad(dy, x, dx, dh=r, dweight=dw, dbias=db, workspace=work.inside)
        assert work.framed()
        outs.append((y, h, dx, dw, db))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("cols", [300, 5000, 20_000])
def test_a_call_in_a_graph(cols):
    """Replayed on other inputs, with eager work between."""
    x, r, dy = (rand(200, cols, F16) for _ in range(3))
    W, B = vector(cols, F32, 1.0), vector(cols, F32, 0.0)
    y, h, dx = (torch.empty(200, cols, dtype=F16, device=DEV) for _ in range(3))
    dw, db = torch.empty(cols, device=DEV), torch.empty(cols, device=DEV)
    work = torch.empty(R.umap_rows_layer_norm_grad_workspace(200, cols), dtype=torch.uint8, device=DEV)

    def step(stream=None):
        R.umap_rows_layer_norm(x, y, weight=W, bias=B, residual=r, h=h, stream=stream)
        R.umap_rows_layer_norm_grad(dy, h, dx, weight=W, dweight=dw, dbias=db, workspace=work, stream=stream)

    step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step(torch.cuda.current_stream())
    for turn in range(4):
        for t in (x, r, dy, W):
            t.normal_(0.2 * turn)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (y, h, dx, dw, db)]
        for t in (y, h, dx, dw, db):
            t.fill_(3.0)
        work.random_(0, 256)
        step()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (y, h, dx, dw, db)))
