"""Balance loss, z loss, counts and their gradient against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _inputs(seed, T, E, K, dt, masked=True, pad=0, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    z = (spread * torch.randn(T, E, generator=g) + torch.randn(E, generator=g)).to(DT[dt])
    ids = torch.stack([torch.randperm(E, generator=g)[:K] for _ in range(T)]).to(torch.int32) if T else torch.empty(0, K, dtype=torch.int32)
    mask = torch.rand(T, generator=g) < 0.8 if masked else None
    if masked and T > 4:
        mask[0], mask[1] = True, False
        z[1] = float("nan")                          # padding rows hold anything
        ids[2, 0] = -1
        ids[3, 0] = E                                # out of range: not counted
        z[4] = -math.inf                             # nothing left
        mask[4] = True
    if pad:
        wide = torch.full((T, E + pad), float("nan"), dtype=z.dtype)
        wide[:, :E] = z
        return wide.to(DEV)[:, :E], z, ids.to(DEV), ids, (mask.to(DEV) if masked else None), mask
    return z.to(DEV), z, ids.to(DEV), ids, (mask.to(DEV) if masked else None), mask


def _formula(z, ids, mask, grad=(0.0, 0.0), extra=None):
    """fp64: loss [2], counts [E], gradient [T][E] by the formula; extra: a perturbation of the logits."""
    z = z.double()
    if extra is not None:
        z = z + extra
    T, E = z.shape
    K = ids.shape[1]
    keep = (z != -math.inf).any(1) if T else torch.zeros(0, dtype=torch.bool)
    if mask is not None:
        keep &= mask
    n = int(keep.sum())
    counts = torch.zeros(E, dtype=torch.int64)
    d = torch.zeros(T, E, dtype=torch.float64)
    if n == 0:
        return torch.zeros(2, dtype=torch.float64), counts, d
    k = ids[keep].reshape(-1).long()
    counts += torch.bincount(k[(k >= 0) & (k < E)], minlength=E)
    zk = z[keep]
    lse = torch.logsumexp(zk, 1)
    p = torch.exp(zk - lse[:, None])
    f = counts.double() / (n * K)
    loss = torch.stack([E * (f * p.mean(0)).sum(), (lse ** 2).mean()])
    d[keep] = grad[0] * E / n * p * (f - (p * f).sum(1, keepdim=True)) + grad[1] * 2 / n * lse[:, None] * p
    return loss, counts, d


def _run(zd, idd, md, grad, **kw):
    f = P.router_balance(zd, idd, mask=md, **kw)
    return f, P.router_balance_backward(zd, f, torch.tensor(grad, dtype=torch.float32, device=DEV), mask=md, **kw)


# A probability is exp2 of a rounded fp32 exponent of magnitude m = |z - max| log2(e) (absolute error at most
# (m + |max| log2 e) 2^-24 for the product and the fused sum, times ln 2), the hardware's exp2 (2^-22), the
# row's sum and reciprocal (a few 2^-24): 2^-19 of the value covers logits up to 30.  A gradient is
# p (gb f + c): p's error and one rounding of each of its terms.
P_TOL = 2.0 ** -19


def _check(f, d, z, ids, mask, grad, dt):
    loss, counts, want = _formula(z, ids, mask, grad)
    assert torch.equal(f["counts"].cpu().long(), counts)
    assert ((f["loss"].double().cpu() - loss).abs() <= 4 * P_TOL * loss.abs() + 1e-30).all()
    T, E = z.shape
    keep = want.abs().sum(1) > 0
    # magnitude of a gradient's terms, row by row
    n = max(1, int(f["rows"].item()))
    size = (abs(grad[0]) * E / n + abs(grad[1]) * 2 / n * (z.double()[keep].logsumexp(1, keepdim=True)).abs())
    prob = torch.softmax(z.double()[keep], 1)
    eps = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}[dt]
    floor = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}[dt]        # fp16: half of the smallest step
    tol = P_TOL * prob * size + eps * want[keep].abs() + floor + 1e-37
    got = d.double().cpu()
    assert ((got[keep] - want[keep]).abs() <= tol).all()
    assert (got[~keep] == 0).all()                                   # rows that do not count


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,E,K", [(1, 2, 1), (1, 1, 1), (7, 8, 2), (61, 64, 6), (33, 60, 4), (100, 128, 8), (257, 255, 9), (64, 256, 32),
                                   (1000, 16, 2), (999, 33, 3), (5000, 9, 1)])
def test_losses_counts_and_gradient(dt, T, E, K):
    zd, z, idd, ids, md, mask = _inputs(T + E, T, E, K, dt, masked=T > 4)
    grad = (1.5 * T, 0.25 * T)                                        # scaled as by a loss scale: fp16 keeps its bits
    f, d = _run(zd, idd, md, grad)
    _check(f, d, z, ids, mask, grad, dt)


@pytest.mark.parametrize("dt,pad", [("f32", 1), ("bf16", 3), ("bf16", 8), ("f16", 5)])
def test_strided_logits_and_gradient(dt, pad):
    zd, z, idd, ids, md, mask = _inputs(5, 77, 40, 3, dt, pad=pad)
    out = torch.full((77, 40 + 5), 3.0, dtype=DT[dt], device=DEV)
    grad = (77.0, 10.0)
    f = P.router_balance(zd, idd, mask=md)
    d = P.router_balance_backward(zd, f, torch.tensor(grad, device=DEV), mask=md, out=out[:, 2:42])
    _check(f, d, z, ids, mask, grad, dt)
    assert (out[:, :2] == 3).all() and (out[:, 42:] == 3).all()


def test_gradient_against_differences():
    """Central differences of the loss in 64 bits (counts held: ids do not move) along random
    directions; the step's own error is O(h^2)."""
    T, E, K = 40, 24, 3
    zd, z, idd, ids, md, mask = _inputs(9, T, E, K, "f32")
    mask[4] = False                                                    # the row of -infinities has no direction
    md = mask.to(DEV)
    for grad in ((1.0, 0.0), (0.0, 1.0), (0.7, 0.3)):
        f, d = _run(zd, idd, md, grad)
        g = torch.Generator().manual_seed(1)
        for _ in range(3):
            v = torch.randn(T, E, generator=g, dtype=torch.float64)
            v[~mask] = 0
            h = 1e-4
            safe = torch.where(mask[:, None], z.double(), torch.zeros(()).double())
            up = (_formula(safe, ids, mask, extra=h * v)[0] * torch.tensor(grad)).sum()
            dn = (_formula(safe, ids, mask, extra=-h * v)[0] * torch.tensor(grad)).sum()
            slope = float(up - dn) / (2 * h)
            scale = float((d.double().cpu().abs() * v.abs()).sum())
            assert abs(float((d.double().cpu() * v).sum()) - slope) <= 1e-5 * scale + 1e-6


def test_nothing_counts():
    z = torch.randn(6, 10, device=DEV)
    ids = torch.zeros(6, 2, dtype=torch.int32, device=DEV)
    f, d = _run(z, ids, torch.zeros(6, dtype=torch.bool, device=DEV), (1.0, 1.0))
    assert (f["loss"] == 0).all() and (f["counts"] == 0).all() and f["rows"].item() == 0 and (d == 0).all()
    f, d = _run(torch.full_like(z, -math.inf), ids, None, (1.0, 1.0))
    assert (f["loss"] == 0).all() and (f["counts"] == 0).all() and (d == 0).all()
    f, d = _run(torch.empty(0, 10, device=DEV), torch.empty(0, 2, dtype=torch.int32, device=DEV), None, (1.0, 1.0))
    assert (f["loss"] == 0).all() and (f["counts"] == 0).all() and d.shape == (0, 10)


def test_lowest_values_infinities_and_nan():
    z = torch.randn(5, 12)
    z[0, :11] = torch.finfo(torch.float32).min          # all but one at the type's lowest value
    z[1, 3:] = -math.inf
    z[2, :] = 88.0
    ids = torch.zeros(5, 1, dtype=torch.int32)
    f, d = _run(z.to(DEV), ids.to(DEV), None, (1.0, 0.5))
    loss, counts, want = _formula(z, ids, None, (1.0, 0.5))
    assert torch.allclose(f["loss"].double().cpu(), loss, rtol=1e-5)
    assert torch.allclose(d.double().cpu(), want, rtol=1e-4, atol=1e-6)
    z[3, 4] = math.inf                                   # as softmax has it: the row and the losses are NaN
    z[4, 4] = math.nan
    f, d = _run(z.to(DEV), ids.to(DEV), None, (1.0, 0.5))
    assert f["loss"].isnan().all() and d[3:].isnan().all() and d[:3].isfinite().all()


def test_repeated_choices_count_each_time():
    ids = torch.tensor([[3, 3, 1], [3, 0, -1]], dtype=torch.int32, device=DEV)
    f = P.router_balance(torch.randn(2, 5, device=DEV), ids)
    assert f["counts"].tolist() == [1, 1, 0, 3, 0]


def test_same_bits_every_time_on_streams_and_replayed():
    zd, _, idd, _, md, _ = _inputs(12, 20000, 64, 4, "bf16")
    g = torch.tensor([1.0, 1.0], device=DEV)
    ref = P.router_balance(zd, idd, mask=md)
    dref = P.router_balance_backward(zd, ref, g, mask=md)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:                                     # calls that overlap have scratch of their own
        f = P.router_balance(zd, idd, mask=md, stream=s)
        got.append((f, P.router_balance_backward(zd, f, g, mask=md, stream=s)))
    torch.cuda.synchronize()
    for f, d in got:
        assert torch.equal(f["loss"], ref["loss"]) and torch.equal(f["counts"], ref["counts"]) and torch.equal(d, dref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f = P.router_balance(zd, idd, mask=md)
        d = P.router_balance_backward(zd, f, g, mask=md)
    zd.mul_(0.5)
    graph.replay()
    torch.cuda.synchronize()
    f2 = P.router_balance(zd, idd, mask=md)
    assert torch.equal(f["loss"], f2["loss"]) and torch.equal(d, P.router_balance_backward(zd, f2, g, mask=md))


def test_more_than_two_billion_logits():
    """2^24 + 5 rows of 132 experts: the last rows against the formulas, the counts as a whole."""
    T, E, K = (1 << 24) + 5, 132, 2
    few = torch.randn(4096, E, generator=torch.Generator().manual_seed(3)).to(DEV).bfloat16()
    z = few.repeat(T // 4096 + 1, 1)[:T]
    ids = torch.arange(T * K, dtype=torch.int64, device=DEV).remainder_(E).to(torch.int32).view(T, K)
    f = P.router_balance(z, ids)
    assert f["rows"].item() == T
    assert torch.equal(f["counts"].long(), torch.bincount(ids.flatten().long(), minlength=E))
    g = torch.tensor([float(T), 0.1 * T], device=DEV)
    d = P.router_balance_backward(z, f, g)
    tail = slice(T - 4, T)
    p = torch.softmax(z[tail].double(), 1)
    share = f["counts"].double() / (T * K)
    lse = torch.logsumexp(z[tail].double(), 1, keepdim=True)
    want = E * p * (share - (p * share).sum(1, keepdim=True)) + 0.2 * lse * p
    size = p * (E * share.max() + 0.2 * lse.abs())
    assert ((d[tail].double() - want).abs() <= P_TOL * size + 2.0 ** -8 * want.abs()).all()
    assert torch.equal(d[:4096], d[4096:8192])               # the same rows, the same gradient
