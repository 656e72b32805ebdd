"""The token-row operators from their definitions, in 64 bits on the CPU, and the error
bounds that follow from the operators' own arithmetic: fp32 from the inputs on, one rounding
to the result's type.  U[type] is half a unit in the last place, relative to the value."""

from __future__ import annotations

import torch

F64 = torch.float64
U = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}
# half the spacing of the smallest values
TINY = {torch.float32: 2.0**-150, torch.float16: 2.0**-25, torch.bfloat16: 2.0**-134}
LARGEST = {torch.int8: 127.0, torch.float8_e4m3fn: 448.0}
E32 = 2.0**-24


def values(x: torch.Tensor, scales=None, group: int = 0) -> torch.Tensor:
    """The numbers that a tensor holds, on the CPU in 64 bits."""
    v = x.cpu().float().to(F64)
    if scales is not None:
        group = group or x.shape[1]
        column = torch.arange(x.shape[1]) // group
        v = v * scales.cpu().to(F64).reshape(x.shape[0], -(-x.shape[1] // group))[:, column]
    return v


def lookup(table64, ids, scale):
    ids = ids.cpu().long()
    there = (ids >= 0) & (ids < table64.shape[0])
    y = torch.zeros((ids.numel(), table64.shape[1]), dtype=F64)
    y[there] = table64[ids[there]] * scale
    return y


def lookup_grad(dout64, ids, rows, scale, start=None):
    """The gradient, and the sum of the terms' magnitudes, which the error goes by."""
    ids = ids.cpu().long()
    there = (ids >= 0) & (ids < rows)
    g = torch.zeros((rows, dout64.shape[1]), dtype=F64)
    m = torch.zeros_like(g)
    g.index_add_(0, ids[there], dout64[there] * scale)
    m.index_add_(0, ids[there], dout64[there].abs() * abs(scale))
    if start is not None:
        g, m = g + start, m + start.abs()
    return g, m


def counts(ids, rows):
    ids = ids.cpu().long()
    return torch.bincount(ids[(ids >= 0) & (ids < rows)], minlength=rows).to(F64)[:, None]


def norm(x64, residual64, weight64, eps):
    h = x64 if residual64 is None else x64 + residual64
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return h, y if weight64 is None else y * weight64


def norm_bound(x64, residual64, weight64, eps, dtype):
    """Bound of |y - exact|: a row's squares are added by 64 threads at least, then their sums."""
    h, y = norm(x64, residual64, weight64, eps)
    parts = x64.abs() + (0 if residual64 is None else residual64.abs())
    rho = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    w = 1 if weight64 is None else weight64.abs()
    steps = (-(-x64.shape[1] // 64) + 24) * E32
    # an error of h also moves its row's norm
    moved = (h.abs() * parts).mean(1, keepdim=True) * rho * rho
    return U[dtype] * y.abs() + steps * y.abs() + 2 * E32 * (parts * rho * w + y.abs() * moved) + TINY[dtype]


def norm_grad(dy64, h64, weight64, eps, dh64=None):
    """dx and dw, and the magnitudes that their errors go by."""
    cols = h64.shape[1]
    rho = 1 / torch.sqrt((h64 * h64).mean(1, keepdim=True) + eps)
    g = dy64 if weight64 is None else dy64 * weight64
    dx = rho * g - h64 * rho**3 * (g * h64).sum(1, keepdim=True) / cols
    size = rho * g.abs() + h64.abs() * rho**3 * (g * h64).abs().sum(1, keepdim=True) / cols
    if dh64 is not None:
        dx, size = dx + dh64, size + dh64.abs()
    t = dy64 * h64 * rho
    return dx, size, t.sum(0), t.abs().sum(0)
