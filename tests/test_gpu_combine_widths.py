"""Combination and its gradients at widths of every kind, with tokens enough for a warp to take four pieces of 256 columns, against 64 bits."""
import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("K", [1, 2, 3, 8])
@pytest.mark.parametrize("yt,ot", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("T,C", [(9600, 512), (9473, 768), (9472, 1024), (5000, 1536), (9500, 300), (3200, 2560), (3157, 2880), (3158, 2881), (2400, 3584), (9471, 1032)])
def test_values_and_gradients(T, C, yt, ot, K):
    dt = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
    g = torch.Generator(device=DEV).manual_seed(T + C + K)
    E, scale = 2 * K + 3, 0.3
    ids = torch.rand(T, E, generator=g, device=DEV).topk(K, 1).indices.to(torch.int32)
    ids[torch.rand(T, K, generator=g, device=DEV) < 0.02] = -1
    plan = P.group_rows(ids.contiguous(), E)
    y = torch.randn(T * K, C, generator=g, device=DEV).to(dt[yt])
    y[int(plan["starts"][E]):] = float("nan")                                  # nobody's
    w = torch.rand(T, K, generator=g, device=DEV)
    w[plan["slots"] < 0] = float("nan")
    res = torch.randn(T, C, generator=g, device=DEV).to(dt[ot])
    grad = torch.randn(T, C, generator=g, device=DEV).to(dt[ot])
    there = plan["slots"] >= 0
    at, share = plan["slots"].clamp(min=0).long(), torch.where(there, scale * w.double(), torch.zeros((), dtype=torch.float64, device=DEV))
    want, size = res.double(), res.double().abs()
    for k in range(K):
        term = torch.where(there[:, k:k + 1], share[:, k:k + 1] * y[at[:, k]].double(), torch.zeros((), dtype=torch.float64, device=DEV))
        want, size = want + term, size + term.abs()
    # a product of scale and weight rounded once, K fused additions; one rounding of the result
    eps, tiny = torch.finfo(dt[ot]).eps / 2, 2. ** -25 if ot == "f16" else 0.
    bound = (K + 2) * 2 ** -24 * size
    bound = bound + eps * (want.abs() + bound) + tiny
    out = P.combine_rows(y, plan, w, residual=res, scale=scale)
    assert ((out.double() - want).abs() <= bound).all()
    mine = res.clone()
    P.combine_rows(y, plan, w, residual=mine, scale=scale, out=mine)
    assert torch.equal(mine, out)
    if ot == yt:
        alone = P.combine_rows(y, plan, w, scale=scale)
        # its one rounding is half a step of its own value, which may be larger than that of the sum with the residual (-1.30 there, 0.35 here)
        bare, off = want - res.double(), (K + 2) * 2 ** -24 * (size - res.double().abs())
        assert ((alone.double() - bare).abs() <= off + eps * (bare.abs() + off) + tiny + 2 ** -50 * size).all()
    dy, dw = P.combine_rows_backward(grad, y, plan, w, scale=scale)
    assert not dy[int(plan["starts"][E]):].any() and not dw[~there].any()
    e16, t16 = torch.finfo(dt[yt]).eps / 2, 2. ** -25 if yt == "f16" else 0.
    for k in range(K):
        on = there[:, k]
        rows, gk = at[:, k][on], grad[on].double()
        d = share[:, k][on][:, None] * gk
        assert ((dy[rows].double() - d).abs() <= (e16 + 2 ** -22) * d.abs() + t16).all()
        yk = y[rows].double()
        # C products added up in fp32, whichever way
        assert ((dw[:, k][on].double() - scale * (gk * yk).sum(1)).abs() <= scale * (C / 8 + 40) * 2 ** -24 * (gk * yk).abs().sum(1)).all()
