"""What the operators that take part in torch's graph refuse: forward-mode derivatives, which they have none of."""
import pytest
import torch
import torch.autograd.forward_ad as fwAD

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def _calls():
    g = torch.Generator(device=DEV).manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    z, ids = rand(40, 8), torch.randint(0, 4, (40, 2), generator=g, device=DEV).to(torch.int32)
    one = torch.randint(0, 3, (40,), generator=g, device=DEV).to(torch.int32)
    plan, ad = P.group_rows(ids, 4), P.group_rows(one, 3)
    x, y, w, h = rand(40, 64).to(BF), rand(80, 64).to(BF), rand(40, 2), rand(40, 64)
    a, b, base = rand(3, 8, 64).to(BF), rand(3, 32, 8).to(BF), rand(40, 32)
    return {
        "balance": (z, lambda t: P.router_balance(t, ids)["loss"], None),
        "select": (z, lambda t: P.router_select(t, 2)["w"], None),
        "dispatch": (x, lambda t: P.dispatch_rows(t, plan), plan),
        "combine y": (y, lambda t: P.combine_rows(t, plan, w), plan),
        "combine w": (w, lambda t: P.combine_rows(y, plan, t, residual=h), plan),
        "combine residual": (h, lambda t: P.combine_rows(y, plan, w, residual=t), plan),
        "lora x": (x, lambda t: P.lora(t, a, b, ad, base=base), ad),
        "lora a": (a, lambda t: P.lora(x, t, b, ad, base=base), ad),
        "lora b": (b, lambda t: P.lora(x, a, t, ad, base=base), ad),
        "lora base": (base, lambda t: P.lora(x, a, b, ad, base=t), ad),
    }


NAMES = ["balance", "select", "dispatch", "combine y", "combine w", "combine residual", "lora x", "lora a", "lora b", "lora base"]


@pytest.mark.parametrize("name", NAMES)
def test_forward_mode_is_refused(name):
    t, call, _ = _calls()[name]
    with fwAD.dual_level():
        with pytest.raises(P.StmoeError, match="forward-mode"):
            call(fwAD.make_dual(t, torch.ones_like(t)))
        call(t)                                 # no tangent: as ever


def test_forward_mode_over_a_gradient_is_refused():
    g = torch.Generator(device=DEV).manual_seed(2)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    ids = torch.randint(0, 3, (40,), generator=g, device=DEV).to(torch.int32)
    plan, z, x, a, b = P.group_rows(ids, 3), rand(40, 8), rand(40, 64).to(BF), rand(3, 8, 64).to(BF), rand(3, 32, 8).to(BF)
    f, hidden, balance = P.router_select(z, 2), rand(40, 8), P.router_balance(z, ids[:, None].contiguous())
    grads = {"balance": (rand(2), lambda t: P.router_balance_backward(z, balance, t)),
             "select": (rand(40, 2), lambda t: P.router_select_backward(z, f, t)),
             "combine": (rand(40, 64).to(BF), lambda t: P.combine_rows_backward(t, x, plan)),
             "lora": (rand(40, 32).to(BF), lambda t: P.lora_backward(t, x, a, b, plan, hidden))}
    with fwAD.dual_level():
        for t, call in grads.values():
            with pytest.raises(P.StmoeError, match="forward-mode"):
                call(fwAD.make_dual(t, torch.ones_like(t)))
            call(t)
