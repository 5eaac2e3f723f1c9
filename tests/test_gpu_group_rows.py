"""Grouping, dispatch and combination of rows against plain indexing and sums in 64 bits."""
import math

import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "u8": torch.uint8}


def _ids(seed, T, K, n, lost=0.1):
    g = torch.Generator().manual_seed(seed)
    share = torch.rand(n, generator=g) ** 3 + 1e-6
    ids = torch.multinomial(share, T * K, replacement=True, generator=g).view(T, K).to(torch.int32) if T else torch.empty(0, K, dtype=torch.int32)
    out = torch.rand(T, K, generator=g)
    ids[out < lost / 2] = -1
    ids[(out >= lost / 2) & (out < lost)] = n + 3
    return ids


def _plan(ids, n):
    flat = ids.reshape(-1).long()
    flat = torch.where((flat >= 0) & (flat < n), flat, torch.full_like(flat, n))
    order = flat.sort(stable=True).indices
    counts = torch.bincount(flat, minlength=n + 1)[:n]
    slots = torch.empty_like(order)
    slots[order] = torch.arange(order.numel())
    slots = torch.where(flat < n, slots, torch.full_like(slots, -1)).view(ids.shape)
    return counts, torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)]), order, slots


@pytest.mark.parametrize("T,K,n", [(0, 2, 4), (1, 1, 1), (1, 8, 256), (3, 2, 1024), (64, 6, 64), (33, 1, 5), (511, 8, 8), (512, 8, 128), (4097, 1, 7),
                                   (4096, 1, 1024), (5000, 4, 256), (70000, 3, 60), (131072, 8, 256), (100003, 1, 1024)])
@pytest.mark.parametrize("lost", [0., 0.3, 1.])
def test_grouping(T, K, n, lost):
    ids = _ids(T + n, T, K, n, lost)
    got = P.group_rows(ids.to(DEV), n)
    for name, want in zip(("counts", "starts", "order", "slots"), _plan(ids, n)):
        assert torch.equal(got[name].cpu().long(), want), name


def test_grouping_of_a_vector_and_one_group_taking_all():
    ids = torch.zeros(9000, dtype=torch.int32)
    got = P.group_rows(ids.to(DEV), 3)
    assert got["slots"].shape == (9000,) and got["counts"].tolist() == [9000, 0, 0]
    assert torch.equal(got["order"].cpu(), torch.arange(9000, dtype=torch.int32))


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16", "u8"])
@pytest.mark.parametrize("T,K,C,pad,off", [(1, 1, 1, 0, 0), (5, 3, 7, 0, 0), (64, 6, 2048, 0, 0), (100, 2, 1413, 0, 0), (100, 2, 1413, 11, 1), (33, 8, 64, 8, 0),
                                           (17, 2, 100, 0, 2), (300, 1, 4096, 16, 0), (40, 4, 130, 1, 1), (9, 2, 20000, 0, 0), (64, 3, 17, 0, 3)])
def test_dispatch(T, K, C, pad, off, dt):
    g = torch.Generator().manual_seed(T + C)
    ids = _ids(C, T, K, 9)
    plan = P.group_rows(ids.to(DEV), 9)
    src = torch.randint(0, 200, (T * (C + pad) + off,), generator=g).to(DT[dt]).to(DEV)
    x = src[off:].view(T, C + pad)[:, :C]
    counts, _, order, _ = _plan(ids, 9)
    n = int(counts.sum())
    want = x.cpu()[order[:n] // K]
    rows = P.dispatch_rows(x, plan)
    assert torch.equal(rows.cpu()[:n], want) and not rows[n:].any()
    buf = torch.full((T * K * (C + pad) + off,), 77, dtype=DT[dt], device=DEV)
    out = buf[off:].view(T * K, C + pad)[:, :C]
    assert P.dispatch_rows(x, plan, out=out) is out
    assert torch.equal(out.cpu()[:n], want) and (out[n:] == 77).all()
    buf2 = buf.clone()
    buf2[off:].view(T * K, C + pad)[:n, :C] = 77
    assert (buf2 == 77).all()                       # nothing between the rows was touched


def _combine_case(seed, T, K, C, dt, res, pad=0, lost=0.1):
    g = torch.Generator().manual_seed(seed)
    ids = _ids(seed, T, K, 7, lost)
    plan = P.group_rows(ids.to(DEV), 7)
    y = torch.randn(T * K, C + pad, generator=g).to(DT[dt])
    n = int((plan["slots"] >= 0).sum())
    y[n:] = math.nan                                # nobody's rows
    w = torch.randn(T, K, generator=g)
    w[plan["slots"].cpu() < 0] = math.nan           # nobody's weights
    r = None if res is None else torch.randn(T, C + pad, generator=g).to(DT[res])
    slots = plan["slots"].cpu().long()
    return plan, slots, y.to(DEV)[:, :C], w, None if r is None else r.to(DEV)[:, :C], n


@pytest.mark.parametrize("dt,res", [("f32", None), ("f32", "f32"), ("bf16", None), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("T,K,C,pad", [(1, 1, 1, 0), (1, 8, 2048, 0), (64, 6, 2048, 0), (100, 2, 1001, 0), (37, 3, 100, 4), (50, 2, 257, 7), (9, 4, 8192, 8), (700, 1, 24, 0)])
def test_combine_and_gradients(T, K, C, pad, dt, res):
    plan, slots, y, w, r, n = _combine_case(T + C, T, K, C, dt, res, pad)
    out = P.combine_rows(y, plan, w.to(DEV), residual=r, scale=0.3)
    there = slots >= 0
    yk = torch.where(there[..., None], y.cpu().double()[slots.clamp(min=0)], torch.zeros((), dtype=torch.float64))    # [T][K][C]
    wk = torch.where(there, w.double(), torch.zeros_like(w.double()))
    terms = 0.3 * wk[..., None] * yk
    base = torch.zeros(T, C, dtype=torch.float64) if r is None else r.cpu().double()
    want, size = base + terms.sum(1), base.abs() + terms.abs().sum(1)
    eps = torch.finfo(out.dtype).eps / 2
    # K + 1 sums, the product of scale and weight and the scale's own rounding: each 2^-24
    assert ((out.cpu().double() - want).abs() <= (K + 4) * 2 ** -24 * size + eps * want.abs() + 2 ** -25 * (out.dtype == torch.float16)).all()
    if r is not None:
        mine = r.clone() if pad == 0 else r
        assert P.combine_rows(y, plan, w.to(DEV), residual=mine, scale=0.3, out=mine) is mine
        assert torch.equal(mine, out)
    grad = torch.randn(T, C, generator=torch.Generator().manual_seed(1)).to(out.dtype)
    dy, dw = P.combine_rows_backward(grad.to(DEV), y, plan, w.to(DEV), scale=0.3)
    gd = grad.double()
    want = torch.zeros(T * K, C, dtype=torch.float64)
    want[slots[there]] = (0.3 * wk[..., None] * gd[:, None])[there]
    assert ((dy.cpu().double() - want).abs() <= (4 * 2 ** -24 + torch.finfo(dy.dtype).eps / 2) * want.abs() + 2 ** -25 * (dy.dtype == torch.float16)).all()
    assert not dy[n:].any()
    prod = 0.3 * gd[:, None] * yk
    assert ((dw.cpu().double() - prod.sum(2)).abs() <= (C + 8) * 2 ** -24 * prod.abs().sum(2)).all()
    assert not dw.cpu()[~there].any()


def test_combine_without_weights_is_the_gradient_of_dispatch():
    ids = _ids(3, 90, 3, 5).to(DEV)
    plan = P.group_rows(ids, 5)
    x = torch.randn(90, 130, device=DEV, requires_grad=True)
    rows = P.dispatch_rows(x, plan)
    c = torch.randn(270, 130, device=DEV)
    (rows * c).sum().backward()
    assert torch.equal(x.grad, P.combine_rows(c, plan))
    # the inner product <dispatch(x), c> = <x, combine(c)>
    assert abs(float((rows.double() * c.double()).sum() - (x.double() * x.grad.double()).sum())) < 1e-3


def test_combine_in_the_graph_with_differences():
    T, K, C = 40, 3, 64
    plan = P.group_rows(_ids(4, T, K, 6).to(DEV), 6)
    g = torch.Generator().manual_seed(7)
    y, w, r = (torch.randn(s, generator=g).to(DEV).requires_grad_(True) for s in ((T * K, C), (T, K), (T, C)))
    c = torch.randn(T, C, generator=g).to(DEV)
    out = P.combine_rows(y, plan, w, residual=r, scale=0.5)
    (out * c).sum().backward()
    assert torch.equal(r.grad, c)
    slots = plan["slots"].long()
    there = (slots >= 0).double()

    def value(s, ey, ew):
        yk = (y.detach().double() + s * ey)[slots.clamp(min=0)]
        return float((0.5 * ((w.detach().double() + s * ew) * there)[..., None] * yk * c.double()[:, None]).sum())
    ey, ew = torch.randn(T * K, C, generator=g).double().to(DEV), torch.randn(T, K, generator=g).double().to(DEV)
    want = (value(1e-3, ey, ew) - value(-1e-3, ey, ew)) / 2e-3           # bilinear: differences are exact
    assert abs(float((y.grad.double() * ey).sum() + (w.grad.double() * ew).sum()) - want) < 1e-3 * (1 + abs(want))


def test_slots_of_other_rows_are_left_out():
    """Slots behind the rows that exist are not followed."""
    L = P.lib()
    x, y = torch.ones(4, 8, device=DEV), torch.ones(3, 8, device=DEV)
    slots = torch.tensor([[0], [5], [-7], [2]], dtype=torch.int32, device=DEV)
    out = torch.zeros(3, 8, device=DEV)
    st = torch.cuda.current_stream().cuda_stream
    assert L.stmoe_dispatch_rows(x.data_ptr(), 32, 32, 4, 1, slots.data_ptr(), None, out.data_ptr(), 3, 32, st) == 0
    assert out.sum(1).tolist() == [8, 0, 8]
    res = torch.zeros(4, 8, device=DEV)
    assert L.stmoe_combine_rows(y.data_ptr(), 0, 8, 3, slots.data_ptr(), None, None, 0, 1.0, 4, 1, 8, res.data_ptr(), 0, 8, st) == 0
    assert res.sum(1).tolist() == [8, 0, 0, 8]


def test_offsets_beyond_32_bits():
    """2^31 and more elements between the first and the last row."""
    T, K, C = 3, 1, 1 << 10
    big = torch.empty((1 << 31) + 4 * C, dtype=torch.bfloat16, device=DEV)
    step = (1 << 30) + 8
    x = big.as_strided((T, C), (step, 1))
    x.copy_(torch.randn(T, C, device=DEV))
    plan = P.group_rows(torch.tensor([2, 0, 1], dtype=torch.int32, device=DEV), 3)
    rows = P.dispatch_rows(x, plan)
    assert torch.equal(rows, x[[1, 2, 0]])
    y = torch.empty_like(big).as_strided((T, C), (step, 1))
    P.dispatch_rows(x, plan, out=y)
    assert torch.equal(y, rows)
    assert torch.equal(P.combine_rows(y, plan), x)


def test_captured_and_replayed():
    T, K, n, C = 6000, 4, 32, 256
    ids = _ids(11, T, K, n).to(DEV)
    x = torch.randn(T, C, device=DEV).bfloat16()
    w = torch.rand(T, K, device=DEV)
    plan = P.group_rows(ids, n)
    want = P.combine_rows(P.dispatch_rows(x, plan), plan, w)
    buf = torch.full_like(ids, -1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p = P.group_rows(buf, n)
        out = P.combine_rows(P.dispatch_rows(x, p), p, w)
    buf.copy_(ids)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(p["order"], plan["order"])
