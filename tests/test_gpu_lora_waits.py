"""Bounded waits of the adapters' tile kernels that run out, by a lowered poll limit (no barrier is broken: the limit alone ends
the waits): the kernels end, what depends on an expired wait is NaN, the rest is as it should be, and the next call with
the default limit is whole."""
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
@pytest.mark.parametrize("T,n,r,I,O", [(700, 3, 16, 512, 1000), (2000, 2, 100, 256, 300)])
@pytest.mark.parametrize("limit", [0, 1, 3])
def test_expired_waits_leave_nan_and_nothing_else(polls, limit, T, n, r, I, O, dt):
    g = torch.Generator(device=DEV).manual_seed(T)
    x, base = torch.randn(T, I, generator=g, device=DEV).to(dt), torch.randn(T, O, generator=g, device=DEV).to(dt)
    a, b = (0.1 * torch.randn(n, r, I, generator=g, device=DEV)).to(dt), torch.randn(n, O, r, generator=g, device=DEV).to(dt)
    ids = torch.randint(-1, n, (T,), generator=g, device=DEV).to(torch.int32)
    plan = P.group_rows(ids, n)
    want = P.lora(x, a, b, plan, base=base)
    assert want.isfinite().all()
    torch.cuda.synchronize()
    polls(limit)
    got = P.lora(x, a, b, plan, base=base)
    torch.cuda.synchronize()
    without = ids < 0
    assert torch.equal(got[without], base[without])
    nan = got.isnan()
    assert torch.equal(got[~nan], want[~nan])
    if limit == 0:
        assert nan[~without].all()
    polls(DEFAULT)
    assert torch.equal(P.lora(x, a, b, plan, base=base), want)
