"""The gradient for the rows that a scaled norm took, against differences of the norm itself."""

import pytest
import torch

import rows_reference as ref
from paper_2008_00325_amd import umap_rows as R
from test_gpu_rows import DEV, F32, norm_grad, rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [5, 64, 300, 2048])
@pytest.mark.parametrize("scale", [1.0, 2.0, 0.125, -3.0])
def test_gradients_of_a_scaled_norm_against_differences(dim, scale):
    """d/de of L = sum dy norm(scale (x + e V) + (r + e Q)): scale dx for x, dx for the residual."""
    torch.manual_seed(dim)
    n = 60
    x, r, w, dy = rand(n, dim, F32), rand(n, dim, F32), rand(1, dim, F32)[0], rand(n, dim, F32)
    h, y = torch.empty(n, dim, device=DEV), torch.empty(n, dim, device=DEV)
    R.umap_rows_norm(x, y, weight=w, residual=r, h=h, scale=scale)
    dr, _ = norm_grad(dy, h, w)
    dx = torch.empty(n, dim, device=DEV)
    R.umap_rows_lookup(dr, None, dx, scale=scale)
    x64, r64, w64, dy64 = ref.values(x), ref.values(r), ref.values(w[None])[0], ref.values(dy)
    V, Q = torch.randn(n, dim, dtype=torch.float64), torch.randn(n, dim, dtype=torch.float64)
    size = ref.norm_grad(dy64, scale * x64 + r64, w64, 1e-6)[1]

    def slope(V, Q):
        def L(e):
            return float((ref.norm(scale * (x64 + e * V), r64 + e * Q, w64, 1e-6)[1] * dy64).sum())

        e = 1e-4   # fourth-order differences: the remainder is about e^4
        return (8 * (L(e) - L(-e)) - (L(2 * e) - L(-2 * e))) / (12 * e)

    def close(got, V, Q, move):
        want = slope(V, Q)
        # h's rounding moves the gradient like a few units in its last place
        assert abs(got - want) <= (dim + 64) * ref.E32 * float((size * move.abs()).sum()) + 1e-7 * abs(want) + 1e-6

    zero = torch.zeros_like(V)
    close(float((ref.values(dx) * V).sum()), V, zero, scale * V)
    close(float((ref.values(dr) * Q).sum()), zero, Q, Q)
