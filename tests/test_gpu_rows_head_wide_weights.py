"""fp16 gradients of rows whose weights lie far apart: the table's gradient of a token that only rows of small weight have anything
to do with is as exact as any other's."""

import pytest
import torch

import rows_head_reference
from paper_2008_00325_amd import umap_rows as R
from test_gpu_rows import BF16, DEV, F16, F32
from test_gpu_rows_head import F64, Case, near

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seed():
    torch.manual_seed(23)
    yield
    torch.cuda.synchronize()


def apart(n, groups, cols, k=0, order=None):
    """Rows of `groups` kinds, each of which gives the other kinds' tokens (20 to a kind) logits of -40 and its own ones of 0."""
    case = Case(n, 20 * groups, cols, F16, k=k, absent=0.0, lean=0.0)
    kind = torch.arange(n, device=DEV) % groups if order is None else order
    kinds = torch.eye(groups, device=DEV)
    case.H[:, :groups] = (kinds[kind]).to(F16)
    case.W[:, :groups] = ((kinds - 1) * 40).repeat_interleave(20, 0).to(F16)
    near_own = torch.randint(0, 20, case.tokens.shape, device=DEV)
    case.tokens = near_own + 20 * (kind[:, None] if k else kind)
    return case, kind


def without_allowance(case, weights64, dscale):
    """The definition's gradients and bounds, the table's without an allowance for weights that fp16 does not hold side by side.
    D is 2^15 times as large as its row's weight, in [1/2, 1) times up to 2^-5, makes it: off by 2^-25 2^-10 2 at most."""
    kept, smallest = dict(rows_head_reference.TINY), 2.0**-25
    rows_head_reference.TINY[F16] = 0.0
    try:
        head = case.head()
        dh, dw, dh_bound, dw_bound = head.grads(F16, weights64, dscale)
        dw_bound = dw_bound()
    finally:
        rows_head_reference.TINY.update(kept)
    g = (dscale * case.scale * weights64.abs())[:, None]
    d_off = g * 2.0**-34
    return (dh, dh_bound + smallest + 1.01 * d_off * case.W.to(F64).abs().sum(0),
            dw, dw_bound + smallest + 1.01 * (d_off * case.H.to(F64).abs()).sum(0))


def check(case, weights, dscale):
    lse = case.loss()[1]
    dh, dw = torch.empty_like(case.H), torch.empty_like(case.W)
    case.grad(lse, dh, dw, weights, dscale)
    want_h, bound_h, want_w, bound_w = without_allowance(case, weights.to(F64), dscale)
    near(dh, want_h, bound_h, "dh")
    near(dw, want_w, bound_w, "dtable")
    return dh, dw


@pytest.mark.parametrize("k", [0, 3])
@pytest.mark.parametrize("power", [-12, -20, -24])
@pytest.mark.parametrize("n", [60, 301, 2200])
def test_tokens_of_rows_of_small_weight(n, power, k):
    case, kind = apart(n, 2, 56, k)
    w = torch.where(kind == 0, 1.0, 2.0**power) * (1 + torch.rand(n, device=DEV))
    # the first kind's tokens within fp16's range, the second's ordinary numbers of it
    check(case, w, 2.0**9)


@pytest.mark.parametrize("k", [0, 3])
@pytest.mark.parametrize("n,cols", [(90, 24), (200, 333), (513, 64), (9001, 40), (1500, 300)])
def test_many_weights_side_by_side(n, cols, k):
    """Nine kinds of rows with weights 2^0 .. 2^-32, in an order of no rule, some without part or of weight 0."""
    kind = torch.randint(0, 9, (n,), device=DEV)
    case, _ = apart(n, 9, cols, k, kind)
    case.tokens[::13] = -1
    w = torch.exp2(-4.0 * kind) * (1 + torch.rand(n, device=DEV)) * torch.where(torch.rand(n, device=DEV) < 0.5, 1.0, -1.0)
    w[::17] = 0.0
    w[::26] = torch.nan   # these are among the rows without part
    used = w.clone()
    used[::13] = 0.0
    lse = case.loss()[1]
    dh, dw = torch.empty_like(case.H), torch.empty_like(case.W)
    for dscale in (1.0, 2.0**20):   # the largest weights' tokens at home in fp16, or the smallest's
        case.grad(lse, dh, dw, w, dscale)
        want_h, bound_h, want_w, bound_w = without_allowance(case, used.to(F64), dscale)
        fits_h, fits_w = (x.abs().max(1).values < 6e4 for x in (want_h, want_w))
        near(dh[fits_h], want_h[fits_h], bound_h[fits_h], "dh")
        near(dw[fits_w], want_w[fits_w], bound_w[fits_w], "dtable")
        assert int(fits_w.sum()) >= 20


def test_the_table_gradient_added_and_in_a_graph():
    """Weights that change from one band to many between replays."""
    kind = torch.randint(0, 5, (700,), device=DEV)
    case, _ = apart(700, 5, 72, 0, kind)
    lse = case.loss()[1]
    w = torch.empty(700, device=DEV)
    dh, dw = torch.empty_like(case.H), torch.zeros_like(case.W)
    work = torch.empty(R.umap_rows_cross_entropy_grad_workspace(*case.sizes()), dtype=torch.uint8, device=DEV)

    def step(stream=None):
        R.umap_rows_cross_entropy_grad(case.H, case.W, case.tokens, lse, work, dh=dh, dtable=dw, dloss=w, dscale=8.0, accumulate=True,
                                       stream=stream)

    w.fill_(1.0)
    step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        step(torch.cuda.current_stream())
    for turn in range(4):
        w.copy_(torch.exp2(-6.0 * turn * kind) * (1 + torch.rand(700, device=DEV)))
        dw.fill_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        replayed = dh.clone(), dw.clone()
        dw.fill_(0.25)
        work.random_(0, 256)
        step()
        assert torch.equal(replayed[0], dh) and torch.equal(replayed[1], dw)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ordinary_weights_of_wider_types(dtype):
    """Their exponents hold weights 2^-100 apart."""
    n = 300
    case = Case(n, 200, 40, dtype, absent=0.0, lean=0.0)
    kind = torch.arange(n, device=DEV) % 2
    case.H[:, 0] = (1.0 - 2.0 * kind).to(dtype)
    case.W[:, 0] = torch.where(torch.arange(200, device=DEV) < 100, 44.0, -44.0).to(dtype)
    case.tokens = (case.tokens % 100) + 100 * kind
    w = torch.where(kind == 0, 2.0**60, 2.0**-20) * (1 + torch.rand(n, device=DEV))
    lse = case.loss()[1]
    dh, dw = torch.empty_like(case.H), torch.empty_like(case.W)
    case.grad(lse, dh, dw, w)
    want_h, want_w, bound_h, bound_w = case.head().grads(dtype, w.to(F64))
    near(dh, want_h, bound_h, "dh")
    near(dw, want_w, bound_w(), "dtable")


@pytest.mark.parametrize("spread", [0, 5, 6, 7, 95, 96, 110])
@pytest.mark.parametrize("n", [250, 8191, 8192, 8193])
def test_places_at_the_bounds_of_bands_and_launches(n, spread):
    """Two kinds of weights, 2^-spread apart: the smaller ones' rows count up to 2^-95 of the largest, beyond which they are not in
    dtable (nor are they in what fp16 holds, unless the largest weight's rows have no gradient there)."""
    case, kind = apart(n, 2, 24)
    w = torch.where(kind == 0, 2.0**60, 2.0 ** (60 - spread)) * torch.ones(n, device=DEV)
    dscale = 2.0 ** (spread - 60)   # the smaller weights are 1
    lse = case.loss()[1]
    dh, dw = torch.empty_like(case.H), torch.empty_like(case.W)
    case.grad(lse, dh, dw, w, dscale)
    ones = torch.ones(n, device=DEV)
    want_h, want_w = torch.empty_like(case.H), torch.empty_like(case.W)
    # the smaller weights' rows alone: the others' probability of their tokens is some 2^-57
    case.tokens[kind == 0] = -1
    case.grad(lse, want_h, want_w, ones)
    assert torch.equal(dh[1::2], want_h[1::2])
    if spread <= 40:
        near(dw[20:], want_w[20:].to(F64), 2.0**-9 * want_w[20:].to(F64).abs() + 2.0**-24 + 2.0 ** (spread - 54) * n, "dtable")
    assert bool(torch.isfinite(dw[20:]).all()) or spread > 60
