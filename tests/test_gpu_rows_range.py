"""Token-row norm and its gradient at the ends of fp32's range, and 8-bit values next to their
half steps, against the definitions."""

import pytest
import torch

import rows_reference as ref
from paper_2008_00325_amd import umap_rows as R
from test_gpu_rows import BF16, DEV, F8, F32, I8, check_norm, near, norm_grad

pytestmark = pytest.mark.gpu


def signs(n, dim):
    return torch.randint(0, 2, (n, dim), device=DEV).float() * 2 - 1


@pytest.mark.parametrize("out", [I8, F8])
@pytest.mark.parametrize("group", [0, 32])
@pytest.mark.parametrize("dim", [5, 40, 300, 2048, 9001, 20001])
def test_norm_into_8_bits_of_the_largest_floats(out, group, dim):
    """Finite values however large are stored as such: |y| from 2^119 to 1.4 2^127."""
    torch.manual_seed(dim)
    for power in (120.0, 125.0, 126.0, 127.0):
        x = signs(5, dim) * (1 + 0.4 * torch.rand(5, dim, device=DEV))   # over their norm: 0.7 .. 1.4
        w = torch.full((dim,), 2.0**power, device=DEV)
        check_norm(x, out, w, group=group)
        check_norm(x.to(BF16), out, w, group=group)


@pytest.mark.parametrize("out", [I8, F8])
@pytest.mark.parametrize("group", [0, 32])
@pytest.mark.parametrize("dim", [4, 7, 64, 256, 512, 1024, 4096, 32768])
def test_8_bit_values_are_the_nearest_to_their_quotients(out, group, dim):
    """Rows of ones have the norm one, so that y is the weight: scale and values have to be those of
    its fp32 quotients, also where they lie next to half a step."""
    torch.manual_seed(dim)
    top = ref.LARGEST[out]
    g = group or dim
    for size in (1.0, 2.0**-90, 2.0**100):
        w = torch.empty(dim)
        for c in range(0, dim, g):
            n = min(g, dim - c)
            most = (1 + torch.rand(1)) * size
            step = most / top   # the group's scale
            if out == I8:
                half = torch.randint(-127, 127, (n,)) + 0.5
            else:   # halfway between two neighbours, of three mantissa bits
                half = (2 * torch.randint(8, 16, (n,)) + 1) * 2.0**torch.randint(-10, 4, (n,))
                half = half * (torch.randint(0, 2, (n,)) * 2 - 1)
            near = half * step
            aside = torch.randint(-1, 2, (n,))   # that value, or its neighbour on either side
            near = torch.where(aside == 0, near, torch.nextafter(near, torch.sign(aside) * float("inf")))
            near[torch.randint(0, n, (1,))] = most
            w[c:c + n] = near
        x = torch.ones(3, dim, device=DEV)
        y = torch.empty(3, dim, device=DEV)
        R.umap_rows_norm(x, y, weight=w.to(DEV), eps=0.0)
        assert torch.equal(y.cpu(), w.expand(3, dim))
        q, scales = torch.empty(3, dim, device=DEV, dtype=out), torch.empty(3, -(-dim // g), device=DEV)
        R.umap_rows_norm(x, q, weight=w.to(DEV), y_scales=scales, group=group, eps=0.0)
        want = torch.stack([w[c:c + g].abs().max() for c in range(0, dim, g)]) / top
        assert torch.equal(scales.cpu(), want.expand_as(scales))
        value = w / want.repeat_interleave(g)[:dim]
        value = value.round() if out == I8 else value.clamp(-top, top).to(F8).float()
        assert torch.equal(q.cpu().float(), value.expand(3, dim))


def smallest(n, dim, size):
    """fp32 rows of up to 7 times `size` (a power of two, from the smallest subnormal on), one of them with a single value."""
    x = (torch.randint(-7, 8, (n, dim)).float() * size)
    x[:, 0] = size
    x[-1, 1:] = 0
    return x.to(DEV)


@pytest.mark.parametrize("dim", [1, 5, 9, 64, 300, 1000, 2048, 9001, 20001, 32768])
@pytest.mark.parametrize("eps", [0.0, 1e-44])
def test_norm_of_the_smallest_rows(dim, eps):
    """Finite rows have finite norms, from the smallest subnormal value on."""
    torch.manual_seed(dim)
    eps = float(torch.tensor(eps))   # as the call takes it
    for power in (-149, -146, -143, -140, -130, -110, -40, -31, -30):
        x = smallest(4, dim, 2.0**power)
        check_norm(x, F32, eps=eps)
        check_norm(x, F32, residual=x, eps=eps)
        check_norm(x, I8, eps=eps)


@pytest.mark.parametrize("dim", [5, 9, 64, 300, 1000, 2048, 9001, 20001, 32768])
def test_norm_grad_of_the_smallest_rows(dim):
    """dx is right wherever it is within fp32's range, 1 / norm within it or not."""
    torch.manual_seed(dim)
    for power in (-149, -146, -143, -140, -130, -110, -40, -31, -30):
        h = smallest(4, dim, 2.0**power)
        dy, w = torch.randn(4, dim, device=DEV) * 2.0**-40, 1 + 0.2 * torch.randn(dim, device=DEV)
        dx, dw = norm_grad(dy, h, w, eps=0.0)
        dx64, size, dw64, dw_size = ref.norm_grad(ref.values(dy), ref.values(h), ref.values(w[None])[0], 0.0)
        steps = (-(-dim // 64) + 40) * ref.E32
        near(dx, dx64, steps * size)
        near(dw[None], dw64[None], (12 * ref.E32 + steps) * dw_size[None])


@pytest.mark.parametrize("dim", [5, 300, 9001])
def test_norm_grad_of_the_largest_rows(dim):
    torch.manual_seed(dim)
    h = signs(4, dim) * (1 + 0.9 * torch.rand(4, dim, device=DEV)) * 2.0**127
    dy = torch.randn(4, dim, device=DEV) * 2.0**40
    dx, _ = norm_grad(dy, h)
    dx64, size, _, _ = ref.norm_grad(ref.values(dy), ref.values(h), None, 1e-6)
    near(dx, dx64, (-(-dim // 64) + 40) * ref.E32 * size + 2.0**-149)
