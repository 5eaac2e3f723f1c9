"""Bounded waits that run out (by a lowered poll limit alone) where the inner dimension is split among the CTAs of a cluster, which add
up one another's sums, and in the gradients: every output is NaN or what it would have been."""
import pytest
import torch

import paper_2606_15453_b200 as P
from paper_2606_15453_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DEFAULT = 1 << 22


@pytest.fixture
def polls():
    yield binding.mx4_poll_limit
    torch.cuda.synchronize()
    binding.mx4_poll_limit(DEFAULT)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,n,r,I,O", [(700, 3, 64, 2048, 264), (2000, 2, 100, 2304, 520), (450, 12, 16, 4097, 1000)])
def test_every_output_is_whole_or_nan(polls, T, n, r, I, O, dt):
    g = torch.Generator(device=DEV).manual_seed(T)
    x, base = torch.randn(T, I, generator=g, device=DEV).to(dt), torch.randn(T, O, generator=g, device=DEV).to(dt)
    a, b = (0.02 * torch.randn(n, r, I, generator=g, device=DEV)).to(dt), (0.1 * torch.randn(n, O, r, generator=g, device=DEV)).to(dt)
    ids = torch.randint(-1, n, (T,), generator=g, device=DEV).to(torch.int32)
    grad = torch.randn(T, O, generator=g, device=DEV).to(dt)
    plan = P.group_rows(ids, n)

    def step(hidden):
        return (P.lora(x, a, b, plan, base=base),) + P.lora_backward(grad, x, a, b, plan, hidden)
    hidden = torch.empty(T, r, device=DEV)
    P.lora(x, a, b, plan, base=base, hidden=hidden)
    want = step(hidden)
    assert all(t.isfinite().all() for t in want)
    without = ids < 0
    for limit in (0, 1, 2, 4, 8, 16, 64):
        torch.cuda.synchronize()
        polls(limit)
        got = step(hidden)
        torch.cuda.synchronize()
        polls(DEFAULT)
        for t, w in zip(got, want):
            nan = t.isnan()
            assert torch.equal(t[~nan], w[~nan]), limit
        assert torch.equal(got[0][without], base[without]) and not got[1][without].any()
        assert torch.equal(got[3], want[3])                 # of hidden and the gradient: no wait in its way
        if limit == 0:
            assert got[0][~without].isnan().all() and got[1][~without].isnan().all()
    for t, w in zip(step(hidden), want):
        assert torch.equal(t, w)
