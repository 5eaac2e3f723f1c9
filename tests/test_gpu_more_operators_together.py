"""Calls of the selection, grouping, combination and adapter operators that overlap, share plans, run in two graphs, or reach far."""
import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _work(seed, T):
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)
    return dict(z=r(T, 256).bfloat16(), bias=0.1 * r(256), x=r(T, 512).bfloat16(), a=(r(6, 24, 512) / 20).bfloat16(), b=(0.1 * r(6, 776, 24)).bfloat16(),
                base=r(T, 776).bfloat16(), ids=torch.randint(-1, 6, (T,), generator=g, device=DEV).to(torch.int32))


def _run(w, stream=None):
    f = P.router_select(w["z"], 8, scores="sigmoid", bias=w["bias"], groups=8, top_groups=4, group_best=2, renorm=True, stream=stream)
    plan = P.group_rows(f["ids"], 256, stream=stream)
    rows = P.dispatch_rows(w["x"], plan, stream=stream)
    mine = P.group_rows(w["ids"], 6, stream=stream)
    y = P.lora(w["x"], w["a"], w["b"], mine, base=w["base"], stream=stream)
    return f["ids"], f["w"], plan["order"], rows, y, P.combine_rows(rows, plan, f["w"], stream=stream)


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("T", [5, 400, 6000])
def test_two_streams_at_once(T):
    w = [_work(s, T) for s in (1, 2)]
    want = [_run(x) for x in w]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in w]
    for _ in range(10):
        got = [_run(x, s) for x, s in zip(w, streams)]
        torch.cuda.synchronize()
        assert all(_same(g, r) for g, r in zip(got, want))


def test_two_graphs_replayed_together_share_nothing():
    w = [_work(s, 3000) for s in (3, 4)]
    want = [_run(x) for x in w]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x in w:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(_run(x))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in w]
    for _ in range(5):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(_same(o, r) for o, r in zip(outs, want))


def test_one_plan_for_two_projections_at_once():
    w = _work(5, 2000)
    plan = P.group_rows(w["ids"], 6)
    want = P.lora(w["x"], w["a"], w["b"], plan, base=w["base"])
    torch.cuda.synchronize()
    s = [torch.cuda.Stream() for _ in range(2)]
    got = [P.lora(w["x"], w["a"], w["b"], plan, base=w["base"], stream=x) for x in s]
    torch.cuda.synchronize()
    assert torch.equal(got[0], want) and torch.equal(got[1], want)


@pytest.mark.parametrize("T,step", [(3, (1 << 30) + 8), (256, (1 << 24) + 8)])
def test_adapter_rows_beyond_32_bits(T, step):
    """2^31 and more elements between the first and the last row, for few rows and for tiles."""
    I, O = 128, 192
    x = torch.empty((T - 1) * step + I, dtype=torch.bfloat16, device=DEV).as_strided((T, I), (step, 1))
    out = torch.empty((T - 1) * step + O, dtype=torch.bfloat16, device=DEV).as_strided((T, O), (step, 1))
    x.copy_(torch.randn(T, I, device=DEV))
    a, b, base = (torch.randn(s, device=DEV).bfloat16() for s in ((1, 16, I), (1, O, 16), (T, O)))
    plan = P.group_rows(torch.zeros(T, dtype=torch.int32, device=DEV), 1)
    want = P.lora(x.contiguous(), a, b, plan, base=base)
    P.lora(x, a, b, plan, base=base, out=out)
    assert torch.equal(out, want)


def test_selection_rows_beyond_32_bits():
    T, E, step = 5, 192, (1 << 30) + 16
    z = torch.empty((T - 1) * step + E, dtype=torch.bfloat16, device=DEV).as_strided((T, E), (step, 1))
    z.copy_(torch.randn(T, E, device=DEV))
    f, g = P.router_select(z, 6), torch.randn(T, 6, device=DEV)
    near = z.contiguous()
    want = P.router_select(near, 6)
    assert torch.equal(f["ids"], want["ids"]) and torch.equal(f["w"], want["w"])
    assert torch.equal(P.router_select_backward(z, f, g), P.router_select_backward(near, want, g))


def test_shared_adapter_expanded_and_its_gradient():
    """One adapter's matrices seen as several: strides of zero, gradients added up."""
    w = _work(6, 300)
    a1, b1 = w["a"][:1].clone().requires_grad_(True), w["b"][:1].clone().requires_grad_(True)
    plan = P.group_rows(w["ids"], 6)
    out = P.lora(w["x"], a1.expand(6, -1, -1), b1.expand(6, -1, -1), plan, base=w["base"])
    one = P.group_rows(torch.where(w["ids"] >= 0, torch.zeros_like(w["ids"]), w["ids"]), 1)
    # the two calls may take different kernels: each is within half a step (2^-8) of the value, and 2^-16 of its terms, some 24 of up to 5 x 0.5
    same = P.lora(w["x"], a1.detach(), b1.detach(), one, base=w["base"]).float()
    assert ((out.detach().float() - same).abs() <= 2 ** -7 * same.abs() + 2 ** -9).all()
    out.sum().backward()
    a2, b2 = a1.detach().clone().requires_grad_(True), b1.detach().clone().requires_grad_(True)
    P.lora(w["x"], a2, b2, one, base=w["base"]).sum().backward()
    # six sums rounded to bf16 and added in bf16 against one
    for p, q in ((a1, a2), (b1, b2)):
        assert (p.grad.float() - q.grad.float()).norm() <= 2 ** -6 * q.grad.float().norm()
