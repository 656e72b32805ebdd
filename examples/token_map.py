"""A map of tokens: vectors learned from text, normalised, kept in 8 bits, and laid out.

The text is synthetic: every token belongs to one topic, a sentence keeps to a topic with some noise, and inside a
topic tokens follow Zipf's law.  Skip-gram with negative samples learns a vector per token (the center's vector is
normalised before it meets the context's); the learned table becomes an 8-bit one, its rows the points of a
neighbourhood graph and of a layout, whose trustworthiness is measured.

    python examples/token_map.py [--tokens 2000] [--steps 400]
"""

from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2008_00325_amd import umap_layout as U  # noqa: E402
from paper_2008_00325_amd import umap_rows as R  # noqa: E402

DEV = "cuda"


class Text:
    """Pairs of tokens that stand in one sentence, and tokens for contrast."""

    def __init__(self, tokens: int, topics: int, noise: float, seed: int):
        self.gen = torch.Generator(device=DEV).manual_seed(seed)
        self.tokens, self.topics, self.noise = tokens, topics, noise
        self.topic_of = torch.arange(tokens, device=DEV) % topics

    def _draw(self, topic: torch.Tensor) -> torch.Tensor:
        u = torch.rand(topic.numel(), generator=self.gen, device=DEV)
        most = self.tokens // self.topics
        rank = (torch.exp(u * torch.log(torch.tensor(most + 1.0))) - 1).long().clamp(0, most - 1)
        return rank * self.topics + topic

    def pairs(self, n: int, negatives: int):
        topic = torch.randint(self.topics, (n,), generator=self.gen, device=DEV)
        stray = torch.rand(n, generator=self.gen, device=DEV) < self.noise
        other = torch.randint(self.topics, (n,), generator=self.gen, device=DEV)
        center, context = self._draw(topic), self._draw(torch.where(stray, other, topic))
        contrast = torch.randint(self.tokens, (n * negatives,), generator=self.gen, device=DEV)
        return center, context, contrast


class Vectors:
    """A token's vector as a center (`table`, through a norm with a weight) and as a context (`out`)."""

    def __init__(self, tokens: int, dim: int, batch: int, negatives: int, seed: int):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        f = dict(device=DEV, dtype=torch.float32)
        self.table = torch.randn(tokens, dim, generator=gen, **f)
        self.out = torch.zeros(tokens, dim, **f)
        self.weight = torch.ones(dim, **f)
        # what a step fills, kept from step to step
        self.h, self.y, self.dh = (torch.empty(batch, dim, **f) for _ in range(3))
        self.o = torch.empty(batch * (1 + negatives), dim, **f)
        self.dweight = torch.empty(dim, **f)
        byte = dict(dtype=torch.uint8, device=DEV)
        self.norm_work = torch.empty(R.umap_rows_norm_grad_workspace(batch, dim), **byte)
        self.work = torch.empty(R.umap_rows_lookup_grad_workspace(batch * (1 + negatives), tokens, dim), **byte)

    def step(self, center, context, contrast, rate: float) -> torch.Tensor:
        """One step of stochastic gradient descent; the loss per pair."""
        n, dim = center.numel(), self.table.shape[1]
        R.umap_rows_lookup(self.table, center, self.h)
        R.umap_rows_norm(self.h, self.y, weight=self.weight)
        others = torch.cat([context, contrast])
        R.umap_rows_lookup(self.out, others, self.o)
        o = self.o.view(-1, n, dim)                       # the context, then the contrasts
        score = (o * self.y).sum(2) * dim**-0.5
        sign = torch.ones_like(score)
        sign[1:] = -1
        loss = -torch.nn.functional.logsigmoid(sign * score).sum(0).mean()
        # d loss / d score, for each pair
        d = (-sign * torch.sigmoid(-sign * score) * dim**-0.5)[:, :, None]
        dy = (d * o).sum(0)
        do = (d * self.y).view(-1, dim)
        R.umap_rows_norm_grad(dy, self.h, self.dh, weight=self.weight, dweight=self.dweight, workspace=self.norm_work)
        # the step lands in the tables' rows that took part
        R.umap_rows_lookup_grad(self.dh, center, self.table, self.work, scale=-rate, accumulate=True)
        R.umap_rows_lookup_grad(do, others, self.out, self.work, scale=-rate, accumulate=True)
        self.weight.sub_(self.dweight, alpha=rate / n)
        return loss

    def in_8_bits(self):
        """The normalised table in 8 bits, and its scales."""
        tokens, dim = self.table.shape
        q = torch.empty(tokens, dim, dtype=torch.int8, device=DEV)
        scales = torch.empty(tokens, 1, device=DEV)
        R.umap_rows_norm(self.table, q, weight=self.weight, y_scales=scales)
        return q, scales


def neighbours(X: torch.Tensor, k: int):
    """Exact k nearest neighbours (ids, distances) of rows."""
    d = (X * X).sum(1)[:, None] + (X * X).sum(1)[None] - 2 * (X @ X.T)
    d.fill_diagonal_(float("inf"))
    d, ids = torch.topk(d, k, largest=False)
    return ids.int().contiguous(), d.clamp(min=0).sqrt().contiguous()


def lay_out(X: torch.Tensor, k: int, epochs: int, seed: int) -> torch.Tensor:
    n = X.shape[0]
    ids, dists = neighbours(X, k)
    rows, cols = (torch.empty(2 * n * k, dtype=torch.int32, device=DEV) for _ in range(2))
    vals = torch.empty(2 * n * k, device=DEV)
    U.umap_fuzzy_graph_device(n, k, ids, dists, rows, cols, vals)
    a, b = U.umap_fit_ab(1.0, 0.1)
    Y = torch.empty(n, 2, device=DEV)
    with U.umap_layout_create_device(n, 2, rows, cols, vals, 2 * n * k, a, b, epochs, 5) as h:
        U.umap_layout_run(h, seed)
        U.umap_layout_get_device(h, Y)
        torch.cuda.synchronize()
    return Y


def run(tokens: int = 2000, topics: int = 10, dim: int = 64, steps: int = 400, batch: int = 8192, negatives: int = 5,
        rate: float = 0.05, k: int = 15, seed: int = 1) -> dict:
    text = Text(tokens, topics, 0.1, seed)
    vectors = Vectors(tokens, dim, batch, negatives, seed + 1)
    losses = [vectors.step(*text.pairs(batch, negatives), rate) for _ in range(steps)]
    q, scales = vectors.in_8_bits()
    X = torch.empty(tokens, dim, device=DEV)
    R.umap_rows_lookup(q, None, X, table_scales=scales)
    Y = lay_out(X, k, 200, seed)
    near, _ = neighbours(Y, k)
    alike = (text.topic_of[near.long()] == text.topic_of[:, None]).float().mean()
    return {"first loss": float(losses[0]), "last loss": float(torch.stack(losses[-10:]).mean()),
            "neighbours of one topic": float(alike), "trustworthiness": U.umap_trustworthiness(X, Y, k), "layout": Y}


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--tokens", type=int, default=2000)
    p.add_argument("--steps", type=int, default=400)
    a = p.parse_args()
    for name, value in run(tokens=a.tokens, steps=a.steps).items():
        if name != "layout":
            print(f"{name}: {value:.4f}")


if __name__ == "__main__":
    main()
