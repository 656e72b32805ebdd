"""A run of the row operators as a model of tokens uses them: rows looked up, a layer norm, the loss against the same
table (tied) or a teacher, and all gradients, against autograd of the same model in 64 bits."""

import pytest
import torch

from paper_2008_00325_amd import umap_rows as R
from test_gpu_rows import BF16, DEV, F32

pytestmark = pytest.mark.gpu
F64 = torch.float64


class Model:
    """Tokens' vectors, a layer norm of them, and the same table as the head."""

    def __init__(self, tokens, dim, n, dtype, k=0):
        gen = torch.Generator(device=DEV).manual_seed(3)
        self.table = (torch.randn(tokens, dim, generator=gen, device=DEV) * dim**-0.5).to(dtype)
        self.weight = 1 + 0.1 * torch.randn(dim, generator=gen, device=DEV)
        self.bias = 0.1 * torch.randn(dim, generator=gen, device=DEV)
        self.x, self.h, self.dh, self.dx = (torch.empty(n, dim, dtype=dtype, device=DEV) for _ in range(4))
        self.dtable = torch.empty_like(self.table)
        self.dweight, self.dbias = (torch.empty(dim, device=DEV) for _ in range(2))
        self.loss, self.lse = (torch.empty(n, device=DEV) for _ in range(2))
        self.scale = dim**0.5
        sizes = (n, tokens, dim) + ((k,) if k else ()) + (dtype,)
        name = "distill" if k else "cross_entropy"
        need = max(getattr(R, f"umap_rows_{name}_workspace")(*sizes), getattr(R, f"umap_rows_{name}_grad_workspace")(*sizes),
                   R.umap_rows_layer_norm_grad_workspace(n, dim), R.umap_rows_lookup_grad_workspace(n, tokens, dim))
        self.work = torch.empty(need, dtype=torch.uint8, device=DEV)   # one after the other on one stream

    def step(self, ids, targets, teacher=None):
        """The loss of each row; gradients in dtable, dweight, dbias."""
        n = ids.numel()
        R.umap_rows_lookup(self.table, ids, self.x, scale=self.scale)
        R.umap_rows_layer_norm(self.x, self.h, weight=self.weight, bias=self.bias)
        if teacher is None:
            R.umap_rows_cross_entropy(self.h, self.table, targets, self.loss, self.lse, self.work)
            R.umap_rows_cross_entropy_grad(self.h, self.table, targets, self.lse, self.work, dh=self.dh, dtable=self.dtable, dscale=1 / n)
        else:
            R.umap_rows_distill(self.h, self.table, targets, teacher, self.loss, self.lse, self.work)
            R.umap_rows_distill_grad(self.h, self.table, targets, teacher, self.lse, self.work, dh=self.dh, dtable=self.dtable, dscale=1 / n)
        R.umap_rows_layer_norm_grad(self.dh, self.x, self.dx, weight=self.weight, dweight=self.dweight, dbias=self.dbias, workspace=self.work)
        R.umap_rows_lookup_grad(self.dx, ids, self.dtable, self.work, scale=self.scale, accumulate=True)
        return self.loss


def batch(n, tokens, k, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    ids = torch.randint(0, tokens, (n,), generator=gen, device=DEV)
    targets = (ids * 7 + 1) % tokens   # what follows a token is certain
    if not k:
        targets[::11] = -1
        return ids, targets, None
    lists = (targets[:, None] + torch.arange(k, device=DEV)) % tokens
    lists[::11] = -1
    return ids, lists, 3.0 - torch.arange(k, device=DEV).float().expand(n, k).contiguous()


@pytest.mark.parametrize("k", [0, 3])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_of_the_whole_model(dtype, k):
    tokens, dim, n = 150, 40, 220
    m = Model(tokens, dim, n, dtype, k)
    ids, targets, teacher = batch(n, tokens, k, 5)
    loss = m.step(ids, targets, teacher).sum().to(F64) / n
    table, weight, bias = (x.to(F64).requires_grad_() for x in (m.table, m.weight, m.bias))
    h = torch.nn.functional.layer_norm(table[ids] * m.scale, (dim,), weight, bias, 1e-5)
    log_p = torch.log_softmax(h @ table.T, 1)
    if k:
        there = targets[:, 0] >= 0
        q = torch.softmax(teacher.to(F64), 1)
        terms = (q * (torch.log(q) - log_p.gather(1, targets.clamp(min=0)))).sum(1)
    else:
        there = targets >= 0
        terms = -log_p.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    want = torch.where(there, terms, 0.0).sum() / n
    want.backward()
    want = want.detach()
    # every stage rounds to the table's type (half a unit in the last place: 2^-8 in bf16), five stages one after the other
    unit = 2.0**-8 if dtype == BF16 else 2.0**-20
    assert abs(float(loss - want)) < 5 * unit * float(want.abs() + 1)
    for got, ref in ((m.dtable, table.grad), (m.dweight, weight.grad), (m.dbias, bias.grad)):
        assert float((got.to(F64) - ref).norm() / ref.norm()) < 5 * unit

