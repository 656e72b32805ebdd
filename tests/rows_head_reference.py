"""The head of the token rows (loss of rows against a table, and its gradient) from its definition in 64
bits, and the error bounds that follow from the operators' own arithmetic: logits, sums and
probabilities in fp32, the entries of D in the inputs' type, one rounding per output.

A sum of n fp32 terms in any order is off by at most n E32 times the sum of their magnitudes, to first order."""

from __future__ import annotations

import math

import torch

from rows_reference import E32, TINY, U

F64 = torch.float64


def shares(ids, rows, teacher64=None, teacher_scale=1.0):
    """Every row's distribution over the table, and whether a row takes part."""
    n = ids.shape[0]
    ids = ids.reshape(n, -1).long()
    there = (ids >= 0) & (ids < rows)
    if teacher64 is None:
        q = there.to(F64)
    else:
        a = (teacher64 * teacher_scale).masked_fill(~there, -math.inf)
        there = a != -math.inf
        most = a.amax(1, keepdim=True)
        e = torch.where(there, torch.exp(a - torch.where(most == -math.inf, 0.0, most)), 0.0)
        q = e / torch.where(there.any(1, keepdim=True), e.sum(1, keepdim=True), 1.0)
    full = torch.zeros((n, rows), dtype=F64, device=ids.device)
    full.scatter_add_(1, torch.where(there, ids, 0), torch.where(there, q, 0.0))
    inner = torch.where(full > 0, full * torch.log(torch.where(full > 0, full, 1.0)), torch.where(full.isnan(), full, 0.0)).sum(1)
    return full, inner, there.any(1)


class Head:
    """h64 (n x cols) against table64 (rows x cols)."""

    def __init__(self, h64, table64, ids, scale=1.0, teacher64=None, teacher_scale=1.0):
        self.h, self.w, self.scale = h64, table64, scale
        self.n, self.rows, self.cols = h64.shape[0], table64.shape[0], h64.shape[1]
        self.q, self.inner, self.part = shares(ids, self.rows, teacher64, teacher_scale)
        self.k = 1 if teacher64 is None else ids.numel() // max(1, self.n)
        # an error of the teacher's logits, as fp32 products and differences
        self.q_err = 0.0 if teacher64 is None else (2 * E32 * (teacher64 * teacher_scale).nan_to_num(0, 0, 0).abs().amax(1) + (self.k + 50) * E32)[:, None]
        self.z = scale * (h64 @ table64.T)
        self.lse = torch.logsumexp(self.z, 1)
        self.p = torch.exp(self.z - self.lse[:, None])
        # products of 16-bit values are exact, fp32's are rounded; then cols terms, times scale
        self.z_err = (self.cols + 3) * E32 * abs(scale) * (h64.abs() @ table64.abs().T)

    def loss(self):
        each = torch.where(self.q > 0, self.q * (self.z - self.lse[:, None]), 0.0).sum(1)
        return torch.where(self.part, self.inner - each, 0.0)

    def lse_bound(self):
        """The logits' errors (a mean of them under p moves lse), and those of the sum of exponentials: every
        exponential is off by its argument's rounding, and sums run over at most 128 of a lane, 8 joins and the tiles."""
        off = self.z_err.amax(1)
        spread = (self.p * (self.z - self.z.amax(1, keepdim=True)).abs()).sum(1)
        steps = 128 + 8 * 4 + self.rows / 128 / 64 * 4 + 64
        return off + (steps + 8 * spread + 4 * self.lse.abs() + 4 * self.z.abs().amax(1)) * E32 + 4e-7

    def loss_bound(self):
        own = torch.where(self.q > 0, self.q * (self.z_err + 4 * E32 * (self.z.abs() + self.lse.abs()[:, None])), 0.0).sum(1)
        size = torch.where(self.q > 0, self.q * (torch.log(self.q.clamp(min=1e-300)).abs() + (self.z - self.lse[:, None]).abs()), 0.0).sum(1)
        q = self.q_err if isinstance(self.q_err, float) else self.q_err[:, 0]
        # shares of zero size in fp32: k times 2^-126 times the distances, far below the rest
        return self.lse_bound() + own + size * (2 * q + (self.k + 10) * E32) + 2 * q

    def grads(self, dtype, dloss64=None, dscale=1.0):
        """dh, dtable and the bounds of their errors."""
        g = dscale * self.scale * (torch.ones(self.n, dtype=F64, device=self.h.device) if dloss64 is None else dloss64)
        part = self.part & (g != 0)
        g = torch.where(part, g, 0.0)[:, None]
        h = torch.where(part[:, None], self.h, 0.0)
        p = torch.where(part[:, None], self.p, 0.0)
        d = g * (p - self.q)
        # p: errors of its logit and of lse, of their difference and of the hardware's exponential
        rel = self.z_err + self.lse_bound()[:, None] + 4 * E32 * (self.z.abs() + self.lse.abs()[:, None]) + 8 * E32
        rel = torch.where(part[:, None], torch.expm1(rel), 0.0)
        q_err = self.q_err if isinstance(self.q_err, float) else torch.where(part[:, None], self.q_err, 0.0)
        err = g.abs() * (p * rel + self.q * q_err * 2 + 4 * E32 * (p + self.q)) + 4 * E32 * d.abs()
        # the hardware's exponential gives 0 where the value lies below fp32's smallest ordinary number, 2^-126: a
        # probability that is lost so is off by less than that
        err = err + g.abs() * 2.0**-126
        err = err + U[dtype] * (d.abs() + err)
        largest = g.abs().max() if self.n else torch.tensor(0.0)
        if dtype == torch.float16:   # D times 2^14 (its row's weight as a number from 1/2 on): half of fp16's smallest step
            err = err + g.abs() * 2 * 2.0**-25 * 2.0**-14
        elif dtype == torch.bfloat16:
            err = err + g.abs() * 2 * 2.0**-134
        dh, dh_size = d @ self.w, (d.abs() + err) @ self.w.abs()
        dh_err = err @ self.w.abs() + (self.rows + 8) * E32 * dh_size
        dw, dw_size = d.T @ h, (d.abs() + err).T @ h.abs()
        dw_err = err.T @ h.abs() + (self.n + 8) * E32 * dw_size
        # a weighted row's h is stored times a power of two at most 1
        lost = TINY[dtype] * 2 * largest * torch.where(part[:, None], p + self.q, 0.0).sum(0)[:, None]
        dw_err = dw_err + (lost if dloss64 is not None else 0.0)

        def rounded(x, e):
            return e + U[dtype] * (x.abs() + e) + TINY[dtype]

        return dh, dw, rounded(dh, dh_err), lambda old=None: rounded(dw if old is None else dw + old, dw_err + (0 if old is None else 2 * E32 * (dw.abs() + old.abs())))
