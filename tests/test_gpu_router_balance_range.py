"""Balance loss, z loss, counts and gradient over the whole range of logits: rows at a mask's fill values, at the
type's lowest and highest, against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2606_15453_b200 as P
from test_gpu_router_balance import P_TOL

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
FLOOR = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}      # fp16: half of its smallest step
F32_MAX = torch.finfo(torch.float32).max


def _ordinary(seed, T, E, K, dt):
    g = torch.Generator().manual_seed(seed)
    z = (2 * torch.randn(T, E, generator=g)).to(DT[dt])
    ids = torch.stack([torch.randperm(E, generator=g)[:K] for _ in range(T)]).to(torch.int32)
    return z, ids


def _formula(z, ids, grad):
    """fp64: loss [2], counts [E], gradient [T][E].  The maximum is subtracted first here too: exp(z - lse)
    would lose log E beside 1e20 even in 64 bits."""
    z = z.double()
    T, E = z.shape
    keep = (z != -math.inf).any(1)
    zk, n = z[keep], int(keep.sum())
    k = ids[keep].reshape(-1).long()
    counts = torch.bincount(k[(k >= 0) & (k < E)], minlength=E)
    p, lse, f = torch.softmax(zk, 1), torch.logsumexp(zk, 1), counts.double() / (n * ids.shape[1])
    loss = torch.stack([E * (f * p.mean(0)).sum(), (lse ** 2).mean()])
    d = torch.zeros(T, E, dtype=torch.float64)
    d[keep] = grad[0] * E / n * p * (f - (p * f).sum(1, keepdim=True)) + grad[1] * 2 / n * lse[:, None] * p
    return loss, counts, d


def _check(z, ids, grad, dt):
    """One row's probabilities are off by P_TOL of their value (exponents that are differences of two logits,
    rounded once, times log2(e), rounded once, for the terms that matter), lse by 2^-24 of its own and 2^-21
    absolute; a gradient by one rounding of its type more."""
    f = P.router_balance(z.to(DEV), ids.to(DEV))
    d = P.router_balance_backward(z.to(DEV), f, torch.tensor(grad, dtype=torch.float32, device=DEV))
    loss, counts, want = _formula(z, ids, grad)
    n = int((z != -math.inf).any(1).sum())
    assert f["rows"].item() == n and torch.equal(f["counts"].cpu().long(), counts)
    got = f["loss"].double().cpu()
    assert abs(got[0] - loss[0]) <= 4 * P_TOL * loss[0]
    if loss[1] <= F32_MAX / 2 and z.double().abs().where(z.isfinite(), torch.zeros(()).double()).max() < 1e18:
        assert abs(got[1] - loss[1]) <= 4 * P_TOL * loss[1] + 2.0 ** -20
    keep = (z != -math.inf).any(1)
    T, E = z.shape
    lse = torch.logsumexp(z.double()[keep], 1, keepdim=True).abs()
    prob = torch.softmax(z.double()[keep], 1)
    tol = P_TOL * prob * (abs(grad[0]) * E / n + abs(grad[1]) * 2 / n * (lse + 1)) + EPS[dt] * want[keep].abs() + FLOOR[dt] + 1e-37
    assert ((d.double().cpu()[keep] - want[keep]).abs() <= tol).all()
    assert (d.double().cpu()[~keep] == 0).all()


VALUES = {"f32": [-F32_MAX, -1e30, -1e20, -1e12, -1e10, -3e9, -1e9, -16777216.0, -1048577.0, -1048576.0, 1048576.0, 1048577.0, 1e9, 1e10, 1e12,
                  1e20, 1e30, 2.4e38, F32_MAX],
          "bf16": [torch.finfo(torch.bfloat16).min, -1e30, -1e20, -1e10, -1e9, 1e9, 1e10, 1e20, torch.finfo(torch.bfloat16).max],
          "f16": [-65504.0, 65504.0]}


@pytest.mark.parametrize("E", [3, 8, 12, 64, 100, 256])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_rows_filled_with_one_value(dt, E):
    """A fully masked row as mask fills write it: uniform probabilities, and the row counts."""
    for v in VALUES[dt]:
        z, ids = _ordinary(E, 9, E, 2, dt)
        z[4] = v
        _check(z, ids, (9.0, 0.0), dt)
        _check(z, ids, (3.0, 0.01), dt)
    for v in VALUES[dt]:
        z, ids = _ordinary(E + 1, 1, E, 1, dt)
        z[:] = v
        _check(z, ids, (1.0, 0.0), dt)


@pytest.mark.parametrize("E", [5, 16, 128])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_one_logit_far_above_or_below_the_others(dt, E):
    for v in VALUES[dt]:
        z, ids = _ordinary(E, 11, E, 1, dt)
        z[2, 1], z[9, E - 1] = v, v
        z[5, :-1] = v
        z[6, 1:] = -math.inf
        z[6, 0] = v
        z[7] = -math.inf
        _check(z, ids, (11.0, 0.0), dt)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_both_ends_of_the_range_in_one_row(dt):
    z, ids = _ordinary(1, 7, 12, 3, dt)
    top = torch.finfo(DT[dt]).max
    z[1, :6], z[1, 6:] = -top, top
    z[3, 0], z[3, 1:] = top, -top
    z[5, 0], z[5, 1:] = 1e10, -1e10
    _check(z, ids, (7.0, 0.0), dt)


def test_large_batch_with_rows_at_fill_values():
    """Several CTAs and the second launch; both losses finite."""
    for dt, fill in (("f32", -1e9), ("bf16", -1e10), ("bf16", torch.finfo(torch.bfloat16).min)):
        z, ids = _ordinary(4, 6000, 64, 4, dt)
        z[::7] = fill
        _check(z, ids, (6000.0, 0.0), dt)


@pytest.mark.parametrize("fill", [-1e19, 1e19, 3e20])
def test_z_loss_is_finite_where_its_mean_is(fill):
    """lse^2 of one row passes the largest fp32 value, its mean over the rows does not."""
    for T in (300, 9000):                                     # one CTA, and many with the second launch
        z, ids = _ordinary(6, T, 16, 2, "f32")
        z[T // 2, :] = fill if abs(fill) < 1e20 else 0.
        z[3, 5] = fill
        loss = _formula(z, ids, (0.0, 0.0))[0]
        got = P.router_balance(z.to(DEV), ids.to(DEV))["loss"].double().cpu()
        if loss[1] < F32_MAX:
            assert abs(got[1] - loss[1]) <= 4 * P_TOL * loss[1]
        else:
            assert got[1] == math.inf
        assert abs(got[0] - loss[0]) <= 4 * P_TOL * loss[0]


@pytest.mark.parametrize("logit", [1.5625, 3.0625, 3.5])
def test_losses_do_not_drift_with_the_tokens(logit):
    """2^28 equal rows; with all of an SM's CTAs at work once, 2362 to a lane.  Added one by one in fp32 their
    probability drifts by 3.2e-5 (the same rounding every time: followed on the CPU).  In groups of 256 rows it may
    drift by 255 2^-24, then 5 additions of lanes, 8 of warps and the store of a CTA's sum, 2^-24 each, on top of
    the probability's own 2^-20 (a row's exponents are below 6, where 2^-22 of exp2 and a few 2^-24 are all there
    is); an lse is off by 2^-21."""
    T, E = 1 << 28, 8
    row = torch.zeros(E, dtype=torch.bfloat16, device=DEV)
    row[0] = logit
    z = row.repeat(T, 1)
    f = P.router_balance(z, torch.zeros(T, 1, dtype=torch.int32, device=DEV))
    p, lse = math.exp(logit) / (math.exp(logit) + 7), math.log(math.exp(logit) + 7)
    assert f["rows"].item() == T and f["counts"].tolist() == [T] + [0] * 7
    got = f["loss"].double().cpu()
    assert abs(got[0] - 8 * p) <= (269 * 2.0 ** -24 + 2.0 ** -20) * 8 * p
    assert abs(got[1] - lse ** 2) <= 2 * lse * 2.0 ** -21 + 2.0 ** -23 * lse ** 2


@pytest.mark.parametrize("grad", [(math.inf, 1.0), (1.0, -math.inf), (math.nan, 1.0), (1.0, math.nan), (math.inf, math.inf)])
@pytest.mark.parametrize("dt,E", [("f32", 12), ("f32", 7), ("bf16", 64), ("f16", 16), ("bf16", 200)])
def test_rows_that_do_not_count_have_zero_gradient_whatever_the_losses_have(dt, E, grad):
    """An overflowed loss scale, for example: padding stays out of what the caller's network sees."""
    z, ids = _ordinary(8, 70, E, 2, dt)
    mask = torch.ones(70, dtype=torch.bool)
    mask[1::3] = False
    z[1] = math.nan
    z[2::9] = -math.inf
    f = P.router_balance(z.to(DEV), ids.to(DEV), mask=mask.to(DEV))
    out = torch.full((70, E), 3.0, dtype=z.dtype, device=DEV)
    P.router_balance_backward(z.to(DEV), f, torch.tensor(grad, device=DEV), mask=mask.to(DEV), out=out)
    counts = mask & (z != -math.inf).any(1)
    assert (out[~counts.to(DEV)] == 0).all()
    assert not out[counts.to(DEV)].isfinite().all()
    f = P.router_balance(z.to(DEV), ids.to(DEV), mask=torch.zeros_like(mask).to(DEV))
    P.router_balance_backward(z.to(DEV), f, torch.tensor(grad, device=DEV), mask=torch.zeros_like(mask).to(DEV), out=out)
    assert (out == 0).all()
