"""Choice of experts where the rounding of fp32 decides if it is let: groups whose two best values nearly cancel."""
import math

import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _groups_of_two_best(z, bias, G, top_groups, K, scores):
    """ids in fp64: groups by the sum of their two best s + bias, the K best of those that stay; equal ones: the lower index."""
    z, bias = z.double(), bias.double()
    s = torch.softmax(z, 1) if scores == "softmax" else 1 / (1 + torch.exp(-z))
    v = s + bias
    T, E = v.shape
    best = v.view(T, G, E // G).sort(2, descending=True).values[:, :, :2].sum(2)
    stay = torch.zeros(T, G, dtype=torch.bool, device=z.device).scatter_(1, best.sort(dim=1, descending=True, stable=True).indices[:, :top_groups], True)
    v = torch.where(stay.repeat_interleave(E // G, 1), v, torch.full_like(v, -math.inf))
    return v.sort(dim=1, descending=True, stable=True).indices[:, :K].sort(1).values.to(torch.int32), best


# groups of two take the general way, groups of eight and sixteen among 192 and 256 experts a warp a row
@pytest.mark.parametrize("large", [0., 30., 1000., 1e5])
@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,G,top_groups,K", [(4, 2, 1, 1), (24, 12, 3, 4), (64, 8, 3, 6), (192, 24, 5, 8), (256, 16, 12, 8), (256, 8, 1, 4)])
def test_sums_that_cancel(E, G, top_groups, K, scores, large):
    """Every second group has biases of +large and -large for its first two members, which are its best, so that their sum is that of two
    scores, as in the group behind it, whose first two have none and whose scores are nearly the same."""
    g = torch.Generator().manual_seed(E + K)
    T, gs = 20000, E // G
    z = torch.randn(T, G, gs, generator=g)
    z[:, 1::2] = z[:, ::2] + 1e-5 * torch.randn(T, G // 2, 1, generator=g)
    z = z.view(T, E).contiguous()
    bias = torch.zeros(G, gs)
    bias[::2, 0], bias[::2, 1], bias[::2, 2:], bias[1::2, 2:] = large, -large, -2 * large, -large
    bias = bias.view(E)
    f = P.router_select(z.to(DEV), K, scores=scores, bias=bias.to(DEV), groups=G, top_groups=top_groups, group_best=2)
    want, _ = _groups_of_two_best(z, bias, G, top_groups, K, scores)
    assert torch.equal(f["ids"].cpu(), want)


def test_a_large_group_beside_a_small_one():
    """The error is the other group's: its members are large, those of the group it is compared with are not."""
    z = torch.tensor([[-0.377855, 1.951048, 0.551829, 0.608678]]).repeat(4, 1)
    z[1:] += torch.tensor([[1e-6], [2e-6], [-1e-6]])
    for bias in ([1000., -1000., 0., 0.], [0., 0., 1000., -1000.]):
        bias = torch.tensor(bias)
        f = P.router_select(z.to(DEV), 2, scores="sigmoid", bias=bias.to(DEV), groups=2, top_groups=1, group_best=2)
        assert torch.equal(f["ids"].cpu(), _groups_of_two_best(z, bias, 2, 1, 2, "sigmoid")[0])


@pytest.mark.parametrize("E", [8, 64, 200, 256])
@pytest.mark.parametrize("scores", ["sigmoid", "softmax"])
def test_scores_that_are_equal_in_64_bits(E, scores):
    """Without a bias the logits decide, with one of zeros the lower index: of groups too, which are ranked by their best."""
    z = torch.full((3, E), -2000.)
    if scores == "sigmoid":                                # all 1 in 64 bits
        z[:, 1], z[:, 3], z[:, E - 1] = 40., 50., 45.
        want, equal = [3, E - 1], [1, 3]
    else:                                                  # 1, and zeros
        z[:, 1], z[:, 3], z[:, E - 1] = 900., 0., 50.
        want, equal = [1, E - 1], [0, 1]
    z, zeros = z.to(DEV), torch.zeros(E, device=DEV)
    for groups, top in ((1, 1), (2, 2)):
        kw = dict(scores=scores, groups=groups, top_groups=top)
        assert P.router_select(z, 2, **kw)["ids"].tolist() == [want] * 3
        assert P.router_select(z, 2, bias=zeros, **kw)["ids"].tolist() == [equal] * 3
    half = dict(scores=scores, groups=2, top_groups=1)
    assert P.router_select(z, 1, **half)["ids"].tolist() == [[want[0]]] * 3
    assert P.router_select(z, 1, bias=zeros, **half)["ids"].tolist() == [[1]] * 3
