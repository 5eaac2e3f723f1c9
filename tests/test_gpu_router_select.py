"""Choice of experts and its gradient against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF = math.inf


def _definition(z, K, scores="softmax", bias=None, groups=1, top_groups=None, group_best=1, renorm=False, scale=1.0, mask=None, grad=None):
    """Row by row in fp64 on the host: ids, w, dlogits."""
    z = z.double().cpu()
    T, E = z.shape
    b = torch.zeros(E, dtype=torch.float64) if bias is None else bias.double().cpu()
    ids = torch.full((T, K), -1, dtype=torch.int32)
    w, d = torch.zeros(T, K, dtype=torch.float64), torch.zeros(T, E, dtype=torch.float64)
    top_groups = top_groups or groups
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        row = z[t]
        nan = bool(row.isnan().any()) or (scores == "softmax" and bool((row == INF).any()))
        if scores == "softmax":
            m = row[~row.isnan()].max() if (~row.isnan()).any() else torch.tensor(0.)
            row_m = row - (m if torch.isfinite(m) else 0)        # first: at 1e38 a logarithm of a sum would drown in the rounding
            logs = row_m - (torch.logsumexp(row_m, 0) if m > -INF else 0)
        else:
            logs = -torch.logaddexp(torch.zeros_like(row), -row)
        s = torch.exp(logs)
        v = s + b
        if bias is None and (group_best == 1 or groups == 1 or top_groups == groups):
            v = row.clone()
        v[(row == -INF) | row.isnan() | v.isnan()] = -INF
        if top_groups < groups:
            gs = E // groups
            tot = [sum(sorted(v[g * gs:(g + 1) * gs].tolist())[::-1][:group_best]) for g in range(groups)]
            tot = [x if x == x else -INF for x in tot]
            stay = sorted(range(groups), key=lambda g: (-tot[g], g))[:top_groups]
            for g in range(groups):
                if g not in stay:
                    v[g * gs:(g + 1) * gs] = -INF
        best = sorted((e for e in range(E) if v[e] > -INF), key=lambda e: (-float(v[e]), e))[:K]
        best = sorted(best)
        n = len(best)
        ids[t, :n] = torch.tensor(best, dtype=torch.int32)
        if nan:
            w[t], d[t] = math.nan, math.nan
            continue
        if not n:
            continue
        share = torch.softmax(logs[best], 0) if renorm else s[best]
        w[t, :n] = scale * share
        if grad is not None:
            g = scale * grad[t, :n].double().cpu()
            mean = (share * g).sum()
            if scores == "softmax":
                if renorm:
                    d[t, best] = share * (g - mean)
                else:
                    d[t] = -s * mean
                    d[t, best] += share * g
            else:
                d[t, best] = share * ((g - mean) if renorm else g) * torch.sigmoid(-row[best])
    return ids, w, d


def _check(z, K, seed=0, **how):
    dev = {k: (v.to(DEV) if isinstance(v, torch.Tensor) else v) for k, v in how.items()}
    zd = z if z.is_cuda else z.to(DEV)
    T, E = z.shape
    grad = torch.randn(T, K, generator=torch.Generator().manual_seed(seed))
    f = P.router_select(zd, K, **dev)
    d = P.router_select_backward(zd, f, grad.to(DEV))
    ids, w, dz = _definition(z, K, grad=grad, **how)
    assert torch.equal(f["ids"].cpu(), ids)
    # an exponential's argument is off by 2^-24 of itself (a logit's distance from the row's largest, or its logarithm of a sigmoid), the
    # exponential, sum and quotient by a few 2^-24 more
    live = z.float()[torch.isfinite(z.float())]
    reach = min(float(live.abs().max()) if live.numel() else 0., 200.)
    rel = (2 * reach + 16) * 2 ** -23
    got = f["w"].cpu().double()
    nan = w.isnan()
    assert torch.equal(got.isnan(), nan)
    scale = abs(how.get("scale", 1.0))
    assert ((got - w).abs()[~nan] <= rel * w.abs()[~nan] + scale * 2 ** -126).all()
    # every term of the gradient is a product of such weights with differences of the incoming gradients
    top = grad.abs().amax(1, keepdim=True).double() * scale * K
    bound = 4 * rel * top + torch.finfo(z.dtype).eps / 2 * dz.abs() + 2 ** -24 * (z.dtype == torch.float16)
    nan = dz.isnan()
    got = d.cpu().double()
    assert torch.equal(got.isnan(), nan)
    assert ((got - dz).abs() <= bound)[~nan].all()
    return f, d


def _logits(seed, T, E, dt, special=True):
    g = torch.Generator().manual_seed(seed)
    z = (2 * torch.randn(T, E, generator=g) + torch.randn(E, generator=g)).to(DT[dt])
    if special and T > 8:
        z[1] = -INF
        z[2, 1:] = -INF
        z[3, E // 2:] = torch.finfo(DT[dt]).min
        z[4] = torch.finfo(DT[dt]).min
        z[5] = 1.5                                       # all equal
        z[6] = (z[6].float() * 8).round().to(DT[dt]) / 8   # many equal ones
        z[7] = 0.
        z[7, ::2] = -0.
    return z


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("E,K", [(1, 1), (2, 2), (7, 3), (8, 8), (9, 2), (16, 16), (33, 5), (64, 6), (96, 32), (100, 8), (128, 8), (129, 1), (255, 7), (256, 8), (256, 32)])
@pytest.mark.parametrize("scores,renorm", [("softmax", False), ("softmax", True), ("sigmoid", False), ("sigmoid", True)])
def test_choice_weights_and_gradient(E, K, dt, scores, renorm):
    _check(_logits(E + K, 37, E, dt), K, scores=scores, renorm=renorm, scale=1.5)


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,K,groups,top,best", [(256, 8, 8, 4, 2), (256, 8, 8, 3, 1), (160, 6, 5, 2, 2), (64, 6, 8, 3, 2), (32, 4, 32, 7, 1), (24, 3, 8, 2, 2),
                                                 (12, 4, 3, 1, 2), (256, 4, 2, 1, 2), (100, 9, 20, 5, 2), (6, 2, 6, 2, 2), (128, 8, 16, 1, 1), (255, 5, 3, 2, 2)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_groups_and_bias(E, K, groups, top, best, scores, dt):
    g = torch.Generator().manual_seed(E + groups)
    bias = 0.1 * torch.randn(E, generator=g)
    for b in (None, torch.zeros(E), bias):
        _check(_logits(E, 41, E, dt), K, scores=scores, bias=b, groups=groups, top_groups=top, group_best=best, renorm=True, scale=2.5)


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_values_next_to_the_border(scores):
    """Biases that undo the scores' differences to a few 2^-24: the order is that of the 64-bit values."""
    g = torch.Generator().manual_seed(5)
    T, E = 48, 64
    z = torch.randn(1, E, generator=g).expand(T, E).clone()
    z += torch.randn(T, E, generator=g) * 2.0 ** torch.randint(-26, -18, (T, 1), generator=g)
    s = torch.softmax(z[0].double(), 0) if scores == "softmax" else torch.sigmoid(z[0].double())
    bias = (0.25 - s).float()
    _check(z, 8, scores=scores, bias=bias, renorm=True)
    _check(z, 8, scores=scores, bias=bias, groups=8, top_groups=4, group_best=2)


@pytest.mark.parametrize("E", [129, 130, 200, 255, 256])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_rows_at_a_fill_value_with_bias(E, scores):
    """Rows of the type's lowest number throughout, or but for a few, where lanes reach past the last expert."""
    g = torch.Generator().manual_seed(E)
    bias = 0.1 * torch.randn(E, generator=g)
    z = torch.full((12, E), torch.finfo(torch.float32).min)
    z[1, :3], z[2, -2:], z[3, E // 2] = 1., 2., 0.
    for renorm in (False, True):
        _check(z, 6, scores=scores, bias=bias, renorm=renorm)
        _check(z, 6, scores=scores, bias=3e38 * torch.sign(bias), renorm=renorm)
    if E in (200, 256):
        _check(z, 6, scores=scores, bias=bias, groups=E // 8, top_groups=3, group_best=2) if E // 8 <= 32 else None


@pytest.mark.parametrize("E,K,groups,top", [(256, 8, 8, 1), (256, 8, 8, 7), (256, 20, 16, 2), (256, 32, 2, 1), (192, 8, 3, 2), (160, 12, 20, 3), (256, 1, 32, 31)])
def test_groups_of_whole_lanes(E, K, groups, top):
    g = torch.Generator().manual_seed(K)
    z = _logits(K, 60, E, "bf16")
    for best in (1, 2):
        for b in (None, 0.1 * torch.randn(E, generator=g)):
            _check(z, K, scores="sigmoid", bias=b, groups=groups, top_groups=top, group_best=best, renorm=True)
            _check(z, K, bias=b, groups=groups, top_groups=top, group_best=best)


def test_masks_padding_and_bias_that_closes_an_expert():
    z = _logits(3, 50, 64, "bf16", special=False)
    mask = torch.rand(50, generator=torch.Generator().manual_seed(1)) < 0.7
    z[~mask] = math.nan
    bias = torch.zeros(64)
    bias[5], bias[6], bias[7] = -INF, math.nan, INF
    f, d = _check(z, 6, scores="sigmoid", bias=bias, mask=mask, renorm=True)
    ids = f["ids"].cpu()
    assert not ((ids == 5) | (ids == 6)).any() and (ids[mask] == 7).any(1).all()
    assert (ids[~mask] == -1).all() and not f["w"].cpu()[~mask].any() and not d.cpu()[~mask].any()


@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_nan_and_infinity_in_rows_that_count(scores, renorm):
    z = _logits(9, 20, 40, "f32", special=False)
    z[2, 7] = math.nan
    z[3, 9] = INF
    z[4, 3], z[4, 4] = INF, INF
    z[6] = math.nan
    _check(z, 5, scores=scores, renorm=renorm)


def test_strides_alignment_and_given_output():
    for dt, E, pad in (("bf16", 64, 3), ("f32", 60, 4), ("f16", 61, 8), ("bf16", 256, 8)):
        wide = torch.full((33, E + pad), math.nan, dtype=DT[dt])
        wide[:, :E] = _logits(1, 33, E, dt)
        for first in (0, 1):
            base = torch.full((33 * (E + pad) + 1,), math.nan, dtype=DT[dt], device=DEV)
            view = base[first:first + 33 * (E + pad)].view(33, E + pad)
            view.copy_(wide)
            _check(view[:, :E], min(E, 6), scores="sigmoid")
            f = P.router_select(view[:, :E], 4)
            out = torch.full((33, E + 5), 7., dtype=DT[dt], device=DEV)
            g = torch.ones(33, 4, device=DEV)
            P.router_select_backward(view[:, :E], f, g, out=out[:, :E])
            assert torch.equal(out[:, :E], P.router_select_backward(view[:, :E], f, g)) and (out[:, E:] == 7).all()


def test_agrees_with_router_topk():
    g = torch.Generator().manual_seed(2)
    h, wr = torch.randn(33, 256, generator=g).to(DEV), torch.randn(60, 256, generator=g).to(DEV)
    for renorm in (False, True):
        r = P.router_topk(h, wr, 4, renorm=renorm)
        f = P.router_select(r["logits"], 4, renorm=renorm)
        assert torch.equal(f["ids"], r["ids"])
        assert (f["w"] - r["w"]).abs().max() < 2e-6


def test_no_rows_and_one_row():
    f = P.router_select(torch.empty(0, 8, device=DEV), 2)
    assert f["ids"].shape == (0, 2)
    assert P.router_select_backward(torch.empty(0, 8, device=DEV), f, torch.empty(0, 2, device=DEV)).shape == (0, 8)
    _check(_logits(4, 1, 256, "f32"), 8, scores="sigmoid", bias=torch.zeros(256), groups=8, top_groups=4, group_best=2, renorm=True, scale=2.5)


def test_autograd_and_differences():
    z = _logits(8, 12, 24, "f32", special=False).to(DEV)
    c = torch.randn(12, 4, generator=torch.Generator().manual_seed(3)).to(DEV)
    for scores in ("softmax", "sigmoid"):
        for renorm in (False, True):
            zz = z.clone().requires_grad_(True)
            f = P.router_select(zz, 4, scores=scores, renorm=renorm, scale=0.7)
            assert not f["ids"].requires_grad
            (f["w"] * c).sum().backward()
            plain = P.router_select_backward(z, P.router_select(z, 4, scores=scores, renorm=renorm, scale=0.7), c)
            assert torch.equal(zz.grad, plain)
            # central differences of the definition in fp64
            e, h = torch.randn(12, 24, generator=torch.Generator().manual_seed(4)).double(), 1e-6
            ids = f["ids"].cpu().long()

            def value(s):
                x = z.double().cpu() + s * h * e
                logs = torch.log_softmax(x, 1) if scores == "softmax" else torch.nn.functional.logsigmoid(x)
                k = logs.gather(1, ids)
                w = torch.softmax(k, 1) if renorm else torch.exp(k)
                return float((0.7 * w * c.double().cpu()).sum())
            want = (value(1) - value(-1)) / (2 * h)
            assert abs(float((zz.grad.double().cpu() * e).sum()) - want) < 1e-4 * (1 + abs(want))


def test_captured_and_replayed_on_another_stream():
    z = _logits(2, 300, 128, "bf16").to(DEV)
    g = torch.randn(300, 8, device=DEV)
    f = P.router_select(z, 8)
    want = f["ids"].clone(), f["w"].clone(), P.router_select_backward(z, f, g)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        P.router_select(z, 8)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    buf = torch.zeros_like(z)
    with torch.cuda.graph(graph):
        c = P.router_select(buf, 8)
        d = P.router_select_backward(buf, c, g)
    buf.copy_(z)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c["ids"], want[0]) and torch.equal(c["w"], want[1]) and torch.equal(d, want[2])
    with torch.cuda.stream(s):
        again = P.router_select(z, 8, stream=s)
    s.synchronize()
    assert torch.equal(again["ids"], want[0]) and torch.equal(again["w"], want[1])


def test_many_rows_agree_with_few():
    z = _logits(6, 70001, 256, "bf16", special=False).to(DEV)
    bias = 0.1 * torch.randn(256, device=DEV)
    how = dict(scores="sigmoid", bias=bias, groups=8, top_groups=4, group_best=2, renorm=True)
    f = P.router_select(z, 8, **how)
    for a in (0, 12345, 69900):
        part = P.router_select(z[a:a + 100], 8, **how)
        assert torch.equal(part["ids"], f["ids"][a:a + 100]) and torch.equal(part["w"], f["w"][a:a + 100])
