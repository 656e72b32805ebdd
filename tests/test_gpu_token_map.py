"""The token map example: training through the row operators, 8-bit rows, layout."""

import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_token_map_learns_and_lays_out():
    import token_map

    r = token_map.run(tokens=1000, topics=8, steps=300, batch=4096)
    # contexts start at zero: every one of the 1 + 5 scores is 0
    assert abs(r["first loss"] - 6 * math.log(2)) < 1e-4
    assert r["last loss"] < 0.8 * r["first loss"]
    # one in eight by chance
    assert r["neighbours of one topic"] > 0.5
    assert r["trustworthiness"] > 0.8
    assert bool(torch.isfinite(r["layout"]).all())


def test_a_training_step_is_the_loss_s_gradient():
    """The step's change of both tables and of the weight against autograd of the same loss in 64 bits."""
    import token_map

    tokens, dim, n, neg, rate = 50, 24, 300, 3, 0.5
    text, v = token_map.Text(tokens, 5, 0.1, 3), token_map.Vectors(tokens, dim, n, neg, 4)
    v.out.normal_()
    start = [x.clone() for x in (v.table, v.out, v.weight)]
    center, context, contrast = text.pairs(n, neg)
    loss = v.step(center, context, contrast, rate)
    table, out, weight = (x.double().cpu().requires_grad_() for x in start)
    h = table[center.cpu()]
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-6) * weight
    o = out[torch.cat([context, contrast]).cpu()].view(-1, n, dim)
    score = (o * y).sum(2) * dim**-0.5
    terms = -torch.nn.functional.logsigmoid(torch.cat([score[:1], -score[1:]]))
    terms.sum().backward()
    assert abs(float(loss) - float(terms.detach().sum(0).mean())) < 1e-5
    # sums of up to n (1 + neg) fp32 terms of size about 1
    for now, was, grad, step in ((v.table, start[0], table.grad, rate), (v.out, start[1], out.grad, rate),
                                 (v.weight, start[2], weight.grad, rate / n)):
        assert float((now.double().cpu() - (was.double().cpu() - step * grad)).abs().max()) < 1e-3
