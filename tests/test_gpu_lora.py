"""Adapters of many requests beside a projection, and their gradients, against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _ids(g, T, n, how):
    if how == "runs":
        cut = torch.sort(torch.rand(max(n - 1, 0), generator=g)).values * T
        ids = torch.searchsorted(cut, torch.arange(T).float() + 0.5).to(torch.int32)
    else:
        ids = torch.randint(-1, n, (T,), generator=g).to(torch.int32)
    if T > 5:
        ids[torch.rand(T, generator=g) < 0.05] = -1
    return ids


def _case(seed, T, n, r, I, O, dt, how="mixed", pad=0):
    g = torch.Generator().manual_seed(seed)
    t = DT[dt]
    x = torch.randn(T, I + pad, generator=g).to(t).to(DEV)[:, :I]
    a = (torch.randn(n, r, I + pad, generator=g) / math.sqrt(I)).to(t).to(DEV)[:, :, :I]
    b = (0.1 * torch.randn(n, O, r + pad, generator=g)).to(t).to(DEV)[:, :, :r]
    base = torch.randn(T, O + pad, generator=g).to(t).to(DEV)[:, :O]
    scale = (0.5 + torch.rand(n, generator=g)).to(DEV)
    ids = _ids(g, T, n, how)
    grad = torch.randn(T, O, generator=g).to(t).to(DEV)
    return x, a, b, base, scale, ids, grad


def _exact(x, a, b, base, scale, ids, grad, alpha, out_dtype, dt):
    """Values and bounds.  h is a sum of I products in fp32 (2^-23 for each addition, whichever way the tensor cores round), held to 2^-16;
    the second sum has r terms per plane; one rounding at the end."""
    f = dict(dtype=torch.float64, device=DEV)
    T, O = base.shape
    n, r, I = a.shape
    eps, tiny = torch.finfo(out_dtype).eps / 2, 2 ** -25 if out_dtype == torch.float16 else 0.
    e16, t16 = torch.finfo(dt).eps / 2, 2 ** -25 if dt == torch.float16 else 0.
    out, bound = base.double().clone(), torch.zeros(T, O, **f)
    dx, bx = torch.zeros(T, I, **f), torch.zeros(T, I, **f)
    da, ba, db, bb = torch.zeros(n, r, I, **f), torch.zeros(n, r, I, **f), torch.zeros(n, O, r, **f), torch.zeros(n, O, r, **f)
    ids = ids.to(DEV)
    for e in range(n):
        at = (ids == e).nonzero()[:, 0]
        if not len(at):
            continue
        X, A, B, G, c = x[at].double(), a[e].double(), b[e].double(), grad[at].double(), alpha * float(scale[e])
        h, u = X @ A.T, G @ B
        hb = (I + 16) * 2 ** -23 * (X.abs() @ A.abs().T) + 2 ** -16 * h.abs()
        ub = (O + 16) * 2 ** -23 * (G.abs() @ B.abs()) + 2 ** -16 * u.abs()
        top = 2.0 ** -24 * h.abs().amax(1, keepdim=True), 2.0 ** -24 * u.abs().amax(1, keepdim=True)    # fp16 planes' last step
        out[at] += c * (h @ B.T)
        bound[at] = abs(c) * ((hb + top[0]) @ B.abs().T + (4 * r + 16) * 2 ** -23 * (h.abs() @ B.abs().T))
        dx[at] = c * (u @ A)
        bx[at] = abs(c) * ((ub + top[1]) @ A.abs() + (4 * r + 16) * 2 ** -23 * (u.abs() @ A.abs()))
        k = (4 * len(at) + 16) * 2 ** -23
        da[e], db[e] = c * (u.T @ X), c * (G.T @ h)
        ba[e] = abs(c) * ((ub + 2.0 ** -24 * u.abs().max()).T @ X.abs() + k * (u.abs().T @ X.abs()))
        bb[e] = abs(c) * (G.abs().T @ (hb + 2.0 ** -24 * h.abs().max()) + k * (G.abs().T @ h.abs()))
    bound += eps * (out.abs() + bound) + 2 ** -23 * base.double().abs() + tiny
    return (out, bound), (dx, bx * (1 + e16) + e16 * dx.abs() + t16), (da, ba * (1 + e16) + e16 * da.abs() + t16), (db, bb * (1 + e16) + e16 * db.abs() + t16)


def _within(got, want, name):
    v, bound = want
    off = (got.double() - v).abs()
    assert not got.isnan().any(), name
    assert (off <= bound).all(), (name, float((off / bound.clamp(min=1e-300)).max()))


SHAPES = [(1, 1, 1, 8, 8), (1, 3, 16, 4096, 4096), (2, 1, 5, 33, 17), (7, 4, 8, 64, 512), (8, 8, 16, 128, 520), (64, 64, 16, 512, 768), (65, 3, 24, 100, 1000),
          (200, 5, 64, 256, 256), (131, 2, 65, 96, 130), (40, 2, 128, 264, 200), (33, 3, 256, 72, 80), (1000, 7, 16, 512, 300), (777, 1, 33, 200, 136), (520, 1024, 4, 32, 40),
          (1500, 2, 8, 40, 1024), (640, 3, 128, 200, 264), (700, 2, 72, 136, 90), (3000, 20, 16, 64, 48), (450, 12, 16, 192, 130)]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("how", ["mixed", "runs"])
@pytest.mark.parametrize("T,n,r,I,O", SHAPES)
def test_values_and_gradients(T, n, r, I, O, how, dt):
    x, a, b, base, scale, ids, grad = _case(T + n + r, T, n, r, I, O, dt, how)
    plan = P.group_rows(ids.to(DEV), n)
    hidden = torch.full((T, r), math.nan, device=DEV)
    out = P.lora(x, a, b, plan, scale=scale, alpha=1.5, base=base, hidden=hidden)
    dx, da, db = P.lora_backward(grad, x, a, b, plan, hidden, scale=scale, alpha=1.5)
    want = _exact(x, a, b, base, scale, ids, grad, 1.5, out.dtype, x.dtype)
    for got, w, name in zip((out, dx, da, db), want, ("out", "dx", "da", "db")):
        _within(got, w, name)
    without = ((ids < 0) | (ids >= n)).to(DEV)
    assert torch.equal(out[without], base[without]) and not dx[without].any() and not hidden[without].any()


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("T,n,r,I,O,pad", [(70, 4, 16, 128, 136, 1), (70, 4, 16, 128, 136, 8), (1100, 2, 20, 96, 72, 3), (5, 2, 7, 31, 29, 5)])
def test_strided_and_unaligned_operands(T, n, r, I, O, pad, dt):
    x, a, b, base, scale, ids, grad = _case(T, T, n, r, I, O, dt, pad=pad)
    plan = P.group_rows(ids.to(DEV), n)
    whole = torch.full((T, O + pad), 5., dtype=x.dtype, device=DEV)
    out = whole[:, :O]
    hidden = torch.empty(T, r, device=DEV)
    assert P.lora(x, a, b, plan, scale=scale, base=base, out=out, hidden=hidden) is out
    want = _exact(x, a, b, base, scale, ids, grad, 1.0, out.dtype, x.dtype)
    _within(out, want[0], "out")
    assert (whole[:, O:] == 5).all()
    for got, w, name in zip(P.lora_backward(grad, x, a, b, plan, hidden, scale=scale), want[1:], ("dx", "da", "db")):
        _within(got, w, name)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("T", [3, 90, 1200])
def test_fp32_result_no_base_and_in_place(T, dt):
    x, a, b, base, scale, ids, grad = _case(T, T, 3, 16, 256, 264, dt)
    plan = P.group_rows(ids.to(DEV), 3)
    base32 = base.float() * 1.001
    want = _exact(x, a, b, base32, scale, ids, grad, 1.0, torch.float32, x.dtype)[0]
    out = P.lora(x, a, b, plan, scale=scale, base=base32)
    assert out.dtype == torch.float32
    _within(out, want, "fp32")
    mine = base32.clone()
    P.lora(x, a, b, plan, scale=scale, base=mine, out=mine)
    assert torch.equal(mine, out)
    alone = P.lora(x, a, b, plan)
    _within(alone, _exact(x, a, b, torch.zeros_like(base), torch.ones_like(scale), ids, grad, 1.0, x.dtype, x.dtype)[0], "alone")
    assert not alone[(ids < 0).to(DEV)].any()


@pytest.mark.parametrize("dt", ["bf16", "f16"])
def test_large_and_small_inner_values(dt):
    """Inner values beyond fp16's range on either side, whose results are within it."""
    x, a, b, base, scale, ids, grad = _case(5, 300, 2, 16, 512, 64, dt)
    big = (x.float() * 200).to(x.dtype), (a.float() * 200).to(x.dtype), (b.float() * 2 ** -12).to(x.dtype)
    small = (x.float() * 2 ** -9).to(x.dtype), (a.float() * 2 ** -9).to(x.dtype), b * 8
    plan = P.group_rows(ids.to(DEV), 2)
    for xs, as_, bs in (big, small):
        hidden = torch.empty(300, 16, device=DEV)
        out = P.lora(xs, as_, bs, plan, scale=scale, base=base * 0, hidden=hidden)
        want = _exact(xs, as_, bs, base * 0, scale, ids, grad, 1.0, out.dtype, out.dtype)
        _within(out, want[0], "out")
        _, _, db = P.lora_backward(grad, xs, as_, bs, plan, hidden, scale=scale)
        fits = want[3][0].abs() < torch.finfo(x.dtype).max / 2
        off = (db.double() - want[3][0]).abs()
        assert (off[fits] <= want[3][1][fits]).all()


def test_infinity_and_nan_stay_in_their_rows():
    x, a, b, base, scale, ids, grad = _case(6, 64, 4, 16, 128, 128, "bf16")
    ids[:] = torch.arange(64) % 4
    plan = P.group_rows(ids.to(DEV), 4)
    clean = P.lora(x, a, b, plan, base=base)
    x2 = x.clone()
    x2[5, 3], x2[17, 100] = math.nan, math.inf
    out = P.lora(x2, a, b, plan, base=base)
    rest = [t for t in range(64) if t not in (5, 17)]
    assert torch.equal(out[rest], clean[rest]) and out[5].isnan().all() and not out[17].isfinite().any()


@pytest.mark.parametrize("T", [1, 8, 300, 1400])
def test_same_bits_every_time_and_rows_apart(T):
    x, a, b, base, scale, ids, grad = _case(8, T, 3, 16, 512, 512, "bf16")
    plan = P.group_rows(ids.to(DEV), 3)
    one = P.lora(x, a, b, plan, scale=scale, base=base)
    assert torch.equal(one, P.lora(x, a, b, plan, scale=scale, base=base))


def test_in_the_graph():
    x, a, b, base, scale, ids, grad = _case(9, 120, 3, 8, 64, 96, "bf16")
    leaves = [t.clone().requires_grad_(True) for t in (x, a, b, base)]
    plan = P.group_rows(ids.to(DEV), 3)
    out = P.lora(leaves[0], leaves[1], leaves[2], plan, scale=scale, base=leaves[3])
    out.backward(grad)
    hidden = torch.empty(120, 8, device=DEV)
    P.lora(x, a, b, plan, scale=scale, base=base, hidden=hidden)
    for got, want in zip(leaves, P.lora_backward(grad, x, a, b, plan, hidden, scale=scale) + (grad,)):
        assert torch.equal(got.grad, want)


def test_gradients_against_differences():
    """Directional differences of the formula in fp64 at fp16 points; exact for each operand by itself up to rounding."""
    x, a, b, base, scale, ids, grad = _case(10, 50, 2, 8, 48, 40, "f16")
    plan = P.group_rows(ids.to(DEV), 2)
    hidden = torch.empty(50, 8, device=DEV)
    P.lora(x, a, b, plan, scale=scale, base=base, hidden=hidden)
    grads = P.lora_backward(grad, x, a, b, plan, hidden, scale=scale)
    at = ids.clamp(min=0).long().to(DEV)
    c = torch.where(ids.to(DEV) >= 0, scale[at], torch.zeros_like(scale[at])).double()

    def value(X, A, B):
        h = torch.einsum("ti,tri->tr", X, A[at])
        return float((c[:, None] * torch.einsum("tr,tor->to", h, B[at]) * grad.double()).sum())
    point = [t.double() for t in (x, a, b)]
    for i in range(3):
        e = torch.randn(point[i].shape, dtype=torch.float64, device=DEV, generator=torch.Generator(device=DEV).manual_seed(i))
        lo, hi = list(point), list(point)
        lo[i], hi[i] = point[i] - e, point[i] + e
        want = (value(*hi) - value(*lo)) / 2           # linear in each
        got = float((grads[i].double() * e).sum())
        assert abs(got - want) <= 2 ** -11 * float((grads[i].double() * e).abs().sum()) + 1e-6


def test_no_rows():
    x, a, b = torch.empty(0, 16, dtype=torch.bfloat16, device=DEV), torch.ones(2, 4, 16, dtype=torch.bfloat16, device=DEV), torch.ones(2, 8, 4, dtype=torch.bfloat16, device=DEV)
    plan = P.group_rows(torch.empty(0, dtype=torch.int32, device=DEV), 2)
    assert P.lora(x, a, b, plan).shape == (0, 8)
    dx, da, db = P.lora_backward(torch.empty(0, 8, dtype=torch.bfloat16, device=DEV), x, a, b, plan, torch.empty(0, 4, device=DEV))
    assert dx.shape == (0, 16) and not da.any() and not db.any()


def test_captured_and_replayed():
    x, a, b, base, scale, ids, grad = _case(12, 600, 4, 16, 256, 256, "bf16")
    plan = P.group_rows(ids.to(DEV), 4)
    want = P.lora(x, a, b, plan, scale=scale, base=base)
    buf = torch.zeros_like(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = P.lora(buf, a, b, plan, scale=scale, base=base)
    buf.copy_(x)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
