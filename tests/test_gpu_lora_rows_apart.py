"""Adapters: what a row holds reaches no other row, and no gradient of another adapter, with either set of kernels."""
import math

import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SIZES = [(64, 4, 16, 128, 128), (300, 4, 16, 256, 264), (1100, 5, 72, 320, 200), (1100, 5, 24, 203, 131), (700, 3, 130, 128, 136), (2500, 2, 64, 2048, 264)]


def _case(T, n, r, I, O, dt, wide=False):
    g = torch.Generator(device=DEV).manual_seed(T + r)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    x, a, b = rand(T, I).to(dt), (rand(n, r, I) / math.sqrt(I)).to(dt), (0.1 * rand(n, O, r)).to(dt)
    base, grad = rand(T, O).to(torch.float32 if wide else dt), rand(T, O).to(dt)
    ids = torch.randint(-1, n, (T,), generator=g, device=DEV).to(torch.int32)
    ids[:3] = torch.tensor([0, 1, n - 1])
    return x, a, b, base, grad, ids


def _step(x, a, b, base, grad, plan):
    hidden = torch.empty(x.shape[0], a.shape[1], device=DEV)
    out = P.lora(x, a, b, plan, base=base, hidden=hidden)
    return (out, hidden) + P.lora_backward(grad, x, a, b, plan, hidden)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("T,n,r,I,O", SIZES)
def test_infinity_and_nan_stay_in_their_rows(T, n, r, I, O, wide, dt):
    x, a, b, base, grad, ids = _case(T, n, r, I, O, dt, wide)
    plan = P.group_rows(ids, n)
    clean = _step(x, a, b, base, grad, plan)
    # two rows of adapter 0 (one in the first tile, one in the last), one without an adapter
    mine = (ids == 0).nonzero()[:, 0]
    bad = [int(mine[0]), int(mine[-1])]
    nobody = int((ids < 0).nonzero()[0, 0])
    x2, g2 = x.clone(), grad.clone()
    x2[bad[0], 3], x2[bad[1], I - 1], x2[nobody] = math.nan, math.inf, math.nan
    g2[nobody] = math.inf
    out, hidden, dx, da, db = _step(x2, a, b, base, g2, plan)
    rest = torch.ones(T, dtype=torch.bool, device=DEV)
    rest[bad] = False
    assert torch.equal(out[rest], clean[0][rest]) and torch.equal(hidden[rest], clean[1][rest])
    assert out[bad[0]].isnan().all() and not out[bad[1]].isfinite().any()
    assert torch.equal(dx, clean[2])                          # of the gradient alone
    assert torch.equal(da[1:], clean[3][1:]) and torch.equal(db[1:], clean[4][1:])
    cols = torch.ones(I, dtype=torch.bool, device=DEV)
    cols[[3, I - 1]] = False
    assert torch.equal(da[0][:, cols], clean[3][0][:, cols]) and not da[0][:, ~cols].isfinite().any()
    # and in the gradient
    g3 = grad.clone()
    g3[bad[0], 0], g3[bad[1], O - 1] = math.nan, math.inf
    _, _, dx, da, db = _step(x, a, b, base, g3, plan)
    assert torch.equal(dx[rest], clean[2][rest]) and torch.equal(da[1:], clean[3][1:]) and torch.equal(db[1:], clean[4][1:])
    assert dx[bad[0]].isnan().all() and not dx[bad[1]].isfinite().any() and not da[0].isfinite().any()
    cols = torch.ones(O, dtype=torch.bool, device=DEV)
    cols[[0, O - 1]] = False
    assert torch.equal(db[0][cols], clean[4][0][cols])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,n,r,I,O", SIZES)
def test_another_row_changes_nothing(T, n, r, I, O, dt):
    x, a, b, base, grad, ids = _case(T, n, r, I, O, dt)
    plan = P.group_rows(ids, n)
    clean = _step(x, a, b, base, grad, plan)
    for row in (0, 1, T // 2, T - 1):
        x2, g2, base2 = x.clone(), grad.clone(), base.clone()
        x2[row], g2[row], base2[row] = 1000., 1000., 1000.    # beyond fp16 as an inner value
        out, hidden, dx, da, db = _step(x2, a, b, base2, g2, plan)
        rest = torch.arange(T, device=DEV) != row
        for got, want in ((out, clean[0]), (hidden, clean[1]), (dx, clean[2])):
            assert torch.equal(got[rest], want[rest])
        others = torch.arange(n, device=DEV) != int(ids[row])
        assert torch.equal(da[others], clean[3][others]) and torch.equal(db[others], clean[4][others])
