"""The head at every tile shape with logits that are exact in fp32 in any order of their sums: what is left of the bounds shows a
single token's logit that a tile leaves out or counts twice."""

import pytest
import torch

from test_gpu_rows import DEV
from test_gpu_rows_head import F64, SHAPES, Case, near

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _seed():
    torch.manual_seed(29)
    yield
    torch.cuda.synchronize()


def whole_numbers(n, rows, cols, dtype, k=0):
    """Elements -1, 0 and 1, a scale of 1/4.  The tokens at both ends of every 64 and the last 70 have logits 3 larger."""
    case = Case(n, rows, cols, dtype, k=k, absent=0.0)
    some = min(1.0, 16 / cols) ** 0.5   # so that 16 of a logit's terms are not 0
    for x in (case.H, case.W):
        x.copy_(torch.where(torch.rand(x.shape, device=DEV) < some, torch.randint(0, 2, x.shape, device=DEV) * 2 - 1, 0))
    edge = torch.arange(rows, device=DEV)
    edge = (edge % 64 == 0) | (edge % 64 == 63) | (edge >= rows - 70)
    case.H[:, 0] = 1
    case.W[:, 0] = torch.where(edge, 12.0, 0.0).to(dtype)
    case.scale = 0.25
    return case, edge


@pytest.mark.parametrize("n,rows,cols,dtype", SHAPES)
def test_exact_logits_at_every_tile_shape(n, rows, cols, dtype):
    for k in (0, 5):
        case, edge = whole_numbers(n, rows, cols, dtype, k)
        ref = case.head()
        ref.z_err.zero_()   # whole numbers below 2^24, and a power of two
        loss, lse = case.loss()
        near(lse, ref.lse, ref.lse_bound(), "lse")
        near(loss, ref.loss(), ref.loss_bound(), "loss")
        # an edge's token left out would show in most rows
        assert float((ref.lse_bound()[:, None] < ref.p[:, edge]).double().mean()) > 0.9
        dh, dw = torch.empty_like(case.H), torch.empty_like(case.W)
        case.grad(lse, dh, dw, None, 1.0)
        want_h, want_w, bound_h, bound_w = ref.grads(dtype)
        near(dh, want_h, bound_h, "dh")
        near(dw, want_w, bound_w(), "dtable")


@pytest.mark.parametrize("n,rows,cols,dtype", SHAPES)
def test_both_gradients_by_columns_of_one_token_or_row(n, rows, cols, dtype):
    """A column that is 1 for a single token t of the table, 0 for the others: dh of it is D's column t; and one that is 1 for a single
    row of h: dtable of it is D's row.  Every 97th token and row are looked at, and both ends."""
    case, _ = whole_numbers(n, rows, cols, dtype)
    tokens = torch.cat([torch.arange(0, rows, 97, device=DEV), torch.tensor([rows - 1], device=DEV)]).unique()
    lines = torch.cat([torch.arange(0, n, 97, device=DEV), torch.tensor([n - 1], device=DEV)]).unique()
    tokens, lines = tokens[-(cols // 2 - 1):], lines[-(cols // 2 - 1):]
    mid = 1 + len(tokens)
    case.W[:, 1:mid + len(lines)] = 0
    case.H[:, 1:mid + len(lines)] = 0
    case.W[tokens, torch.arange(1, mid, device=DEV)] = 1
    case.H[lines, torch.arange(mid, mid + len(lines), device=DEV)] = 1
    _, lse = case.loss()
    dh, dw = torch.empty_like(case.H), torch.empty_like(case.W)
    case.grad(lse, dh, dw, None, 1.0)
    ref = case.head()
    ref.z_err.zero_()
    want_h, want_w, bound_h, bound_w = ref.grads(dtype)
    near(dh, want_h, bound_h, "dh")
    near(dw, want_w, bound_w(), "dtable")
    # those columns have one term each: without the bounds' allowance for their sums
    rel = ref.lse_bound() + 8 * 2.0**-24 * (1 + ref.lse.abs() + ref.z.abs().amax(1))
    half = torch.finfo(dtype).eps / 2
    d = case.scale * (ref.p - ref.q)
    off = case.scale * (ref.p + ref.q) * rel[:, None] + 2.1 * half * d.abs() + 2.0**-37
    near(dh[:, 1:mid], d[:, tokens], off[:, tokens] + 2.0**-25, "dh, one token")
    near(dw[:, mid:mid + len(lines)], d[lines].T, off[lines].T + 2.0**-25, "dtable, one row")
