"""Balance losses as steps of torch's graph: the gradient that reaches the logits."""
import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _problem(T=300, E=24, K=3, dt=torch.float32, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = torch.randn(T, E, generator=g, device=DEV).to(dt)
    ids = z.float().topk(K, 1).indices.to(torch.int32)
    mask = torch.rand(T, generator=g, device=DEV) < 0.8
    return z, ids, mask


def _direct(z, ids, mask, grad):
    f = P.router_balance(z.detach(), ids, mask=mask)
    return f, P.router_balance_backward(z.detach(), f, grad, mask=mask)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("masked", [False, True])
def test_backward_has_the_gradient_kernels_bits(dt, masked):
    z, ids, mask = _problem(dt=dt)
    mask = mask if masked else None
    z.requires_grad_()
    f = P.router_balance(z, ids, mask=mask)
    assert f["loss"].requires_grad and not f["counts"].requires_grad and not f["rows"].requires_grad
    (f["loss"] * torch.tensor([30.0, 0.5], device=DEV)).sum().backward()
    ref, want = _direct(z, ids, mask, torch.tensor([30.0, 0.5], device=DEV))
    assert torch.equal(z.grad, want) and torch.equal(f["loss"], ref["loss"]) and torch.equal(f["counts"], ref["counts"])
    assert f["rows"].item() == ref["rows"].item() and f["top_k"] == 3


def test_gradient_adds_to_that_of_the_network():
    """Logits of a linear router that also weigh an output: against torch's own formula in 64 bits."""
    g = torch.Generator(device=DEV).manual_seed(5)
    T, H, E, K = 200, 32, 16, 2
    x = torch.randn(T, H, generator=g, device=DEV)
    w = torch.randn(E, H, generator=g, device=DEV).requires_grad_()
    v = torch.randn(E, generator=g, device=DEV)
    z = x @ w.t()
    ids = z.detach().topk(K, 1).indices.to(torch.int32)
    f = P.router_balance(z, ids)
    (f["loss"][0] + 0.1 * f["loss"][1] + (torch.softmax(z, 1) @ v).mean()).backward()
    wd = w.detach().double().requires_grad_()
    zd = x.double() @ wd.t()
    p, lse = torch.softmax(zd, 1), torch.logsumexp(zd, 1)
    share = f["counts"].double() / (T * K)
    (E * (share * p.mean(0)).sum() + 0.1 * (lse ** 2).mean() + (p @ v.double()).mean()).backward()
    # fp32 sums of T = 200 products and what they are made of: 2^-15 of the largest is room for all of it
    assert ((w.grad.double() - wd.grad).abs() <= 2.0 ** -15 * wd.grad.abs().max()).all()


def test_strided_logits_of_a_wider_leaf():
    z, ids, mask = _problem()
    wide = torch.zeros(300, 40, device=DEV)
    wide[:, 5:29] = z
    wide.requires_grad_()
    P.router_balance(wide[:, 5:29], ids, mask=mask)["loss"].sum().backward()
    # the bits of the same rows: those of contiguous ones are read, and added, in another order
    _, want = _direct(wide[:, 5:29], ids, mask, torch.ones(2, device=DEV))
    assert torch.equal(wide.grad[:, 5:29], want) and (wide.grad[:, :5] == 0).all() and (wide.grad[:, 29:] == 0).all()


def test_one_loss_alone_and_a_broadcast_gradient():
    z, ids, mask = _problem()
    z.requires_grad_()
    P.router_balance(z, ids, mask=mask)["loss"][1].backward()
    assert torch.equal(z.grad, _direct(z, ids, mask, torch.tensor([0.0, 1.0], device=DEV))[1])
    z.grad = None
    P.router_balance(z, ids, mask=mask)["loss"].mean().backward()     # an expanded gradient
    assert torch.equal(z.grad, _direct(z, ids, mask, torch.tensor([0.5, 0.5], device=DEV))[1])


def test_no_graph_where_none_is_recorded():
    z, ids, mask = _problem()
    assert P.router_balance(z, ids, mask=mask)["loss"].grad_fn is None
    z.requires_grad_()
    with torch.no_grad():
        assert P.router_balance(z, ids, mask=mask)["loss"].grad_fn is None


def test_explicit_backward_still_takes_logits_that_require_a_gradient():
    z, ids, mask = _problem()
    g = torch.tensor([1.0, 2.0], device=DEV)
    want = _direct(z, ids, mask, g)[1]
    z.requires_grad_()
    f = P.router_balance(z, ids, mask=mask)
    d = P.router_balance_backward(z, f, g, mask=mask)
    assert torch.equal(d, want) and d.grad_fn is None


def test_changed_logits_and_second_derivatives_are_refused():
    z, ids, mask = _problem()
    z.requires_grad_()
    a = z * 1.0
    loss = P.router_balance(a, ids, mask=mask)["loss"].sum()
    a.detach().zero_()                                            # in place, seen by the version counter
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    loss = P.router_balance(z, ids, mask=mask)["loss"].sum()
    (d,) = torch.autograd.grad(loss, z, create_graph=True)
    with pytest.raises(RuntimeError):
        d.sum().backward()


def test_on_another_stream():
    z, ids, mask = _problem(T=20000)
    z.requires_grad_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    f = P.router_balance(z, ids, mask=mask, stream=s)
    with torch.cuda.stream(s):
        total = f["loss"].sum()
        total.backward()
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(z.grad, _direct(z, ids, mask, torch.ones(2, device=DEV))[1])


def test_captured_and_replayed():
    z, ids, mask = _problem(T=5000)
    z.requires_grad_()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):                                     # warm-up as torch asks for it
        torch.autograd.grad(P.router_balance(z, ids, mask=mask)["loss"].sum(), z)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = P.router_balance(z, ids, mask=mask)["loss"]
        (d,) = torch.autograd.grad(loss.sum(), z)
    for seed in (2, 3):
        z2, ids2, mask2 = _problem(T=5000, seed=seed)
        with torch.no_grad():
            z.copy_(z2), ids.copy_(ids2), mask.copy_(mask2)
        graph.replay()
        f, want = _direct(z2, ids2, mask2, torch.ones(2, device=DEV))
        assert torch.equal(d, want) and torch.equal(loss.detach(), f["loss"])


def test_no_tokens():
    z = torch.empty(0, 8, device=DEV, requires_grad=True)
    f = P.router_balance(z, torch.empty(0, 2, dtype=torch.int32, device=DEV))
    f["loss"].sum().backward()
    assert (f["loss"] == 0).all() and z.grad.shape == (0, 8)
