"""Probabilities of the rows' own tokens: a gradient's entry p - q there may nearly cancel, and so may the lse - z of a row of one
token, where the logit rounds as the one does that lse is of.  The rows here have partial sums in the thousands, whose rounding (some 1e-4)
shows in a logit that is added in another order, and logits of about one."""

import math

import pytest
import torch

from rows_reference import E32, U
from test_gpu_rows import BF16, DEV, F16, F32, FLOATS
from test_gpu_rows_head import F64, Case, near

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seed():
    torch.manual_seed(19)
    yield
    torch.cuda.synchronize()


def nearly_cancelling(n, cols, dtype):
    """Rows of h (n x cols) and a vector of `cols`, whose products' sum is far below its halves'."""
    half = cols // 2
    h, w = (1 + torch.rand(n, half, device=DEV)).to(dtype), (1 + torch.rand(half, device=DEV)).to(dtype)
    h = torch.cat([h, h.flip(1), torch.zeros(n, cols - 2 * half, device=DEV, dtype=dtype)], 1)
    more = torch.where(torch.rand(half, device=DEV) < 0.01, 1 + 2.0**-6, 1.0)
    w = torch.cat([w, -(w.flip(0).float() * more).to(dtype), torch.zeros(cols - 2 * half, device=DEV, dtype=dtype)])
    return h, w


@pytest.mark.parametrize("k", [0, 1, 3, 20])
@pytest.mark.parametrize("n,cols", [(1, 2048), (40, 2049), (300, 2048), (2100, 2056)])
@pytest.mark.parametrize("dtype", FLOATS)
def test_a_certain_token_has_no_loss_and_no_gradient(dtype, n, cols, k):
    """A table of one token: lse is its logit z, log 1 being 0, p = 1 = q.  The loss is 0 (of rows
    of one token; others' own logits are dot products of their own).  In 16 bits z counts in units of log 2
    (x), and lse, which is kept in natural ones, is two products and a rounding away each way: x is off by 5 E32 of it,
    and the exponential by 4 E32, so p by (5 |z| + 4) E32 2."""
    case = Case(n, 1, cols, dtype, k=k, absent=0.0)
    case.H, w = nearly_cancelling(n, cols, dtype)
    case.W = w[None].contiguous()
    if k:
        case.tokens[:, 1:] = -1
    for scale in (1.0, 0.5):
        case.scale = scale
        loss, lse = case.loss()
        assert k > 1 or not bool(loss.any())
        assert float(lse.abs().max()) < 60 * scale
        for weights in (None, torch.rand(n, device=DEV) + 0.1):
            dh, dw = torch.full_like(case.H, 7.0), torch.full_like(case.W, 7.0)
            case.grad(lse, dh, dw, weights)
            g = scale * (torch.ones(n, device=DEV) if weights is None else weights).to(F64)[:, None]
            off = 0.0 if dtype == F32 else 2 * (5 * lse.abs().to(F64)[:, None] + 4) * E32 * g
            near(dh, torch.zeros_like(dh, dtype=F64), 1.01 * off * case.W.abs().to(F64) + 2.0**-25, "dh")
            if dtype == F32:
                assert not bool(dh.any()) and not bool(dw.any())
            else:
                near(dw, torch.zeros_like(dw, dtype=F64), 1.01 * (off * case.H.abs().to(F64)).sum(0) + 2.0**-25, "dtable")


@pytest.mark.parametrize("k", [0, 2, 12])
@pytest.mark.parametrize("n", [30, 300, 2100])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_a_nearly_certain_token(dtype, n, k):
    """300 tokens with logits of 0 but the row's own one with 15, where 1 - p is 9.1e-5: dh along that token's vector.

    The own logit in fp32 is off by up to cols E32 times its terms' sum, which moves 1 - p by that factor; lse, about
    15, by 3e-6 of its own rounding, 0.033 of 1 - p."""
    cols, rows = 2048, 300
    case = Case(n, rows, cols, dtype, k=k, absent=0.0)
    h, w = nearly_cancelling(n, cols, dtype)
    w[cols // 2:] = -w[:cols // 2].flip(0)   # now exactly 0
    h[:, [0, cols - 1]], w[0], w[cols - 1] = 1.0, 0.0, 15.0
    case.H, case.W = h.contiguous(), torch.zeros(rows, cols, dtype=dtype, device=DEV)
    case.W[170] = w
    if k:
        case.tokens[:] = -1
        case.tokens[:, k - 1] = 170
    else:
        case.tokens[:] = 170
    loss, lse = case.loss()
    dh = torch.empty_like(case.H)
    case.grad(lse, dh, None)
    rest = (rows - 1) / (rows - 1 + math.exp(15.0))   # 1 - p
    terms = (h.to(F64).abs() * w.to(F64).abs()).sum(1).max()
    moved = math.expm1(cols * E32 * float(terms)) + 0.033
    want = -rest * w.to(F64)
    bound = (moved + 3 * U[dtype]) * want.abs() + 2.0**-25
    near(dh, want.expand_as(dh), bound.expand_as(dh), "dh")
    if k < 2:
        near(loss, torch.full((n,), -math.log1p(-rest), dtype=F64, device=DEV), torch.tensor(rest * moved, device=DEV), "loss")


@pytest.mark.parametrize("ids", [torch.int32, torch.int64])
@pytest.mark.parametrize("k", [0, 1])
@pytest.mark.parametrize("n,rows,cols", [(70, 1_100_003, 7), (1300, 1_100_003, 7), (300, 2_100_000, 64)])
def test_tokens_in_every_piece_and_turn(n, rows, cols, k, ids):
    """Tables of several copied pieces (odd rows, over 128 MB of copies) and rows in several turns: the loss of whole numbers' exact
    logits, from each row's own token wherever it lies."""
    case = Case(n, rows, cols, BF16, k=k, ids=ids, absent=0.2)
    case.H.copy_(torch.randint(-1, 2, case.H.shape, device=DEV))
    case.W.copy_(torch.randint(-1, 2, case.W.shape, device=DEV))
    ends = torch.tensor([0, 63, 64, 255, rows // 2, 1 << 20, (1 << 20) - 1, rows - 1, rows - 2], device=DEV)
    case.tokens.view(-1)[:9] = ends.to(ids)
    loss, lse = case.loss()
    tokens = case.tokens.view(-1).long()
    for first in range(0, n, 100):
        part = slice(first, min(n, first + 100))
        z = case.H[part].float() @ case.W.float().T   # whole numbers
        want = torch.logsumexp(z.to(F64), 1)
        # 300 additions, and exponentials and logits of at most 64, in fp32
        off = (300 + 8 * 64) * E32 + 4e-7
        near(lse[part], want, torch.full_like(want, off), "lse")
        there = (tokens[part] >= 0) & (tokens[part] < rows)
        own = z.gather(1, torch.where(there, tokens[part], 0)[:, None])[:, 0].to(F64)
        near(loss[part], torch.where(there, want - own, 0.0), torch.full_like(want, 2 * off), "loss")


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("n", [20, 300])
def test_rows_that_are_not_finite(n, dtype):
    case = Case(n, 400, 40, dtype, absent=0.0)
    clean = case.loss()
    case.H[3, 5] = math.nan
    case.H[11, 0] = math.inf
    loss, lse = case.loss()
    ok = torch.ones(n, dtype=torch.bool, device=DEV)
    ok[[3, 11]] = False
    assert torch.equal(loss[ok], clean[0][ok]) and torch.equal(lse[ok], clean[1][ok])
    assert math.isnan(float(loss[3])) and math.isnan(float(lse[3])) and not math.isfinite(float(lse[11]))
    dh = torch.empty_like(case.H)
    case.grad(lse, dh, None)
    assert bool(torch.isfinite(dh[ok]).all()) and bool(dh[3].isnan().all())
