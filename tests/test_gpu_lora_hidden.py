"""The inner values that lora hands out (hidden), in every form of the call and with either set of kernels."""
import math

import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("how", ["in place", "in place, fp32", "apart", "no base"])
@pytest.mark.parametrize("T,n,r,I,O", [(1, 2, 16, 64, 64), (3, 2, 16, 64, 64), (90, 4, 16, 256, 1100), (90, 4, 200, 256, 1100), (900, 3, 64, 256, 300), (900, 3, 130, 96, 600)])
def test_rows_without_an_adapter_get_zeros(T, n, r, I, O, how, dt):
    g = torch.Generator().manual_seed(T + r)
    x = torch.randn(T, I, generator=g).to(dt).to(DEV)
    a, b = (torch.randn(n, r, I, generator=g) / math.sqrt(I)).to(dt).to(DEV), (0.1 * torch.randn(n, O, r, generator=g)).to(dt).to(DEV)
    ids = torch.randint(-1, n + 1, (T,), generator=g).to(torch.int32)      # n: outside, as -1 is
    ids[0] = -1
    base = None if how == "no base" else torch.randn(T, O, generator=g).to(torch.float32 if "fp32" in how else dt).to(DEV)
    was = None if base is None else base.clone()
    plan = P.group_rows(ids.to(DEV), n)
    hidden = torch.full((T, r), math.nan, device=DEV)
    out = P.lora(x, a, b, plan, base=base, out=base if "in place" in how else None, hidden=hidden)
    without = ((ids < 0) | (ids >= n)).to(DEV)
    assert not hidden[without].any()                                       # NaN is true
    assert torch.equal(out[without], torch.zeros_like(out[without]) if was is None else was[without])
    at = ids.clamp(0, n - 1).long().to(DEV)
    h = torch.einsum("ti,tri->tr", x.double(), a.double()[at])
    # I products added up in fp32: 2^-23 of their magnitudes for each addition, whichever way the tensor cores round
    bound = (I + 16) * 2 ** -23 * torch.einsum("ti,tri->tr", x.double().abs(), a.double().abs()[at])
    assert ((hidden.double() - h).abs() <= bound)[~without].all()
