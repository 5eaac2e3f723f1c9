"""The operators together: a routed layer of 4-bit experts over many tokens, with an adapter for each request."""
import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _layer(h, wr, bias, gate, up, down, adapters, a, b, K):
    """Router to residual: choice by groups, grouping, dispatch, 4-bit products with adapters beside gate, combination."""
    E, n = wr.shape[0], a.shape[0]
    r = P.router_topk(h, wr, K)
    f = P.router_select(r["logits"], K, scores="sigmoid", bias=bias, groups=4, top_groups=2, group_best=2, renorm=True, scale=2.0)
    plan = P.group_rows(f["ids"], E)
    x = (h * r["inv_rms"][:, None]).bfloat16()
    rows = P.dispatch_rows(x, plan)
    q = P.mx4_quantize(rows)
    g, u = P.mx4_matmul(q, gate, plan["counts"]), P.mx4_matmul(q, up, plan["counts"])
    mine = P.group_rows(P.dispatch_rows(adapters[:, None], plan)[:, 0].contiguous(), n)      # a row's request goes where the row goes
    g = P.lora(rows, a, b, mine, base=g, out=g)
    y = P.mx4_matmul(P.mx4_quantize(torch.nn.functional.silu(g.float()) * u.float()), down, plan["counts"])
    return f, plan, rows, g, u, y, P.combine_rows(y, plan, f["w"], residual=h, scale=0.1)


def _operands(T, E, H, I, n, r, K):
    gen = torch.Generator().manual_seed(T)
    h, wr = torch.randn(T, H, generator=gen).to(DEV), (0.1 * torch.randn(E, H, generator=gen)).to(DEV)
    bias = (0.05 * torch.randn(E, generator=gen)).to(DEV)

    def experts(rows, cols):
        q = P.mx4_quantize((0.05 * torch.randn(E * rows, cols, generator=gen)).to(DEV))
        return q[0].view(E, rows, -1), q[1].view(E, rows, -1)
    gate, up, down = experts(I, H), experts(I, H), experts(H, I)
    adapters = torch.randint(-1, n, (T,), generator=gen).to(torch.int32).to(DEV)
    a, b = (torch.randn(n, r, H, generator=gen) / 16).bfloat16().to(DEV), (0.1 * torch.randn(n, I, r, generator=gen)).bfloat16().to(DEV)
    return h, wr, bias, gate, up, down, adapters, a, b, K


@pytest.mark.parametrize("T", [1, 5, 64])
def test_layer_against_the_definition(T):
    E, H, I, n, r, K = 16, 256, 128, 5, 16, 4
    args = _operands(T, E, H, I, n, r, K)
    h, wr, bias, gate, up, down, adapters, a, b, _ = args
    f, plan, rows, g, u, y, out = _layer(*args)
    total = int(plan["starts"][-1])
    assert total == T * K
    wide = [P.mx4_dequantize(c.reshape(-1, c.shape[2]), s.reshape(-1, s.shape[2]), s.shape[2] * 32).double().view(E, c.shape[1], -1) for c, s in (gate, up, down)]
    xq = P.mx4_dequantize(*P.mx4_quantize(rows), H).double()
    pair = plan["order"].long()
    expert = f["ids"].reshape(-1).long()[pair]
    token = pair // K
    assert torch.equal(rows, (h * P.router_topk(h, wr, K)["inv_rms"][:, None]).bfloat16()[token])
    gate_want = torch.einsum("th,tih->ti", xq, wide[0][expert])
    ad = adapters.long()[token]
    inner = torch.einsum("th,trh->tr", rows.double(), a.double()[ad.clamp(min=0)])
    gate_want += torch.where(ad[:, None] >= 0, torch.einsum("tr,tir->ti", inner, b.double()[ad.clamp(min=0)]), torch.zeros_like(gate_want))
    # two roundings to bf16, of the product and of its sum with the adapter's part, and fp32 sums of 256 and 16 terms
    size = torch.einsum("th,tih->ti", xq.abs(), wide[0].abs()[expert]) + gate_want.abs()
    assert ((g.double() - gate_want).abs() <= 2 ** -8 * (gate_want.abs() + (gate_want - g.double()).abs() + size * 2 ** -2) + 2 ** -12 * size).all()
    act = P.mx4_dequantize(*P.mx4_quantize(torch.nn.functional.silu(g.float()) * u.float()), I).double()
    want_y = torch.einsum("ti,thi->th", act, wide[2][expert])
    assert ((y.double() - want_y).abs() <= 2 ** -8 * want_y.abs() + 2 ** -14 * torch.einsum("ti,thi->th", act.abs(), wide[2].abs()[expert])).all()
    want = h.double()
    want = want.index_add(0, token, 0.1 * f["w"].double().reshape(-1)[pair][:, None] * y.double())
    assert ((out.double() - want).abs() <= 2 ** -20 * (want.abs() + 1)).all()
    assert (f["w"].sum(1) - 2).abs().max() < 1e-5


def test_layer_captured_and_replayed_with_other_tokens():
    args = _operands(48, 16, 256, 128, 5, 16, 4)
    want = _layer(*args)[-1]
    buf = torch.randn_like(args[0])
    _layer(buf, *args[1:])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _layer(buf, *args[1:])[-1]
    buf.copy_(args[0])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_training_step_of_a_router_and_its_adapters():
    """Gradients of router weights and adapters through selection, dispatch, adapters and combination, against torch's own of the same
    formulas in fp64 with the choice held."""
    T, E, H, O, K, n, r = 96, 8, 64, 48, 2, 3, 4
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(T, H, generator=gen).half().to(DEV)
    wr = (0.2 * torch.randn(E, H, generator=gen)).to(DEV).requires_grad_(True)
    a, b = ((0.2 * torch.randn(s, generator=gen)).half().to(DEV).requires_grad_(True) for s in ((E, r, H), (E, O, r)))
    c = torch.randn(T, O, generator=gen).half().to(DEV)
    logits = x.float() @ wr.t()
    f = P.router_select(logits, K, renorm=True)
    plan = P.group_rows(f["ids"], E)
    rows = P.dispatch_rows(x, plan)
    y = P.lora(rows, a, b, P.group_rows(f["ids"].reshape(-1)[plan["order"].long()], E))      # an expert is its adapter
    out = P.combine_rows(y, plan, f["w"])
    out.backward(c)
    W, A, B = (t.detach().double().requires_grad_(True) for t in (wr, a, b))
    ids = f["ids"].long()
    w = torch.softmax((x.double() @ W.t()).gather(1, ids), 1)
    h = torch.einsum("th,tkrh->tkr", x.double(), A[ids])
    (torch.einsum("tk,tkr,tkor->to", w, h, B[ids]) * c.double()).sum().backward()
    # fp16 results and gradients pass three roundings of 2^-11 on the way, of terms that partly cancel: norms within 2^-8
    for got, want in ((wr, W), (a, A), (b, B)):
        assert (got.grad.double() - want.grad).norm() <= 2 ** -8 * want.grad.norm()
