"""Weights of choices whose scores lie far below the others', among few and among many experts."""
import math

import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("E", [8, 64, 128, 160, 256])
@pytest.mark.parametrize("top", [3., -0.5, -20., -39., -45., -90., -1e4])
def test_renormalised_sigmoid_weights(E, top):
    """K logits of a row are the only ones left: the first at `top`, the others down to 130 below it."""
    K, T = 6, 64
    g = torch.Generator().manual_seed(E)
    z = torch.full((T, E), -math.inf)
    at = torch.stack([torch.randperm(E, generator=g)[:K] for _ in range(T)])
    z.scatter_(1, at, top - 130 * torch.rand(T, K, generator=g) * (torch.arange(K) > 0))
    if E > 128:                                   # finite fills far below: an infinity would send the row the general way
        z = torch.where(z == -math.inf, torch.full_like(z, top - 1000.), z)
    f = P.router_select(z.to(DEV), K, scores="sigmoid", renorm=True)
    want = z.gather(1, f["ids"].cpu().long()).double()
    assert torch.equal(f["ids"].cpu().sort(1).values.long(), at.sort(1).values)
    w = torch.softmax(-torch.logaddexp(torch.zeros_like(want), -want), 1)
    # the argument of an exponential is off by 2^-24 of itself, the rest by a few 2^-24; below 2^-126 numbers have fewer bits
    rel = (2 * (130 + min(abs(top), 200.)) + 16) * 2 ** -23 if top > -1000 else (4 * abs(top) + 16) * 2 ** -23
    assert ((f["w"].cpu().double() - w).abs() <= rel * w + 2 ** -126).all()


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("scale", [1e-39, -1e-42, 0., 1e38])
@pytest.mark.parametrize("E", [6, 200])
def test_gradients_at_extreme_scales(E, scale, renorm, scores):
    """Any finite scale: weights and gradients are its multiples, with no more bits than so small a number has."""
    g = torch.Generator().manual_seed(E)
    z, grad = torch.randn(50, E, generator=g).to(DEV), 0.1 * torch.rand(50, 3, generator=g).to(DEV)
    kw = dict(scores=scores, renorm=renorm)
    f, one = P.router_select(z, 3, scale=scale, **kw), P.router_select(z, 3, **kw)
    d, d1 = P.router_select_backward(z, f, grad), P.router_select_backward(z, one, grad)
    assert torch.equal(f["ids"], one["ids"]) and d.isfinite().all()
    s = float(torch.tensor(scale))
    assert ((f["w"].double() - s * one["w"].double()).abs() <= 2 ** -22 * abs(s) + 2 ** -149).all()
    # every gradient is at most the sum of the incoming ones times |scale|; what a scale below 2^-126 leaves of it is below that, too
    assert ((d.double() - s * d1.double()).abs() <= 2 ** -20 * abs(s) + (abs(s) if abs(s) < 2 ** -126 else 0)).all()
