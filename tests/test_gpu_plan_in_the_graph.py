"""Plans between a call and its gradient: what the gradient reads of them may not be written meanwhile."""
import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def _calls():
    g = torch.Generator(device=DEV).manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    ids = torch.randint(0, 4, (40, 2), generator=g, device=DEV).to(torch.int32)
    one = torch.randint(0, 3, (40,), generator=g, device=DEV).to(torch.int32)
    plan, ad = P.group_rows(ids, 4), P.group_rows(one, 3)
    x, y, w = rand(40, 64).to(BF), rand(80, 64).to(BF), rand(40, 2)
    a, b, base = rand(3, 8, 64).to(BF), rand(3, 32, 8).to(BF), rand(40, 32)
    return {
        "dispatch": (x, lambda t: P.dispatch_rows(t, plan), plan),
        "combine y": (y, lambda t: P.combine_rows(t, plan, w), plan),
        "combine w": (w, lambda t: P.combine_rows(y, plan, t), plan),
        "lora x": (x, lambda t: P.lora(t, a, b, ad, base=base), ad),
        "lora a": (a, lambda t: P.lora(x, t, b, ad, base=base), ad),
        "lora b": (b, lambda t: P.lora(x, a, t, ad, base=base), ad),
    }


NAMES = ["dispatch", "combine y", "combine w", "lora x", "lora a", "lora b"]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("what", ["slots", "order", "counts", "starts", "ids"])
def test_a_plan_overwritten_before_its_gradient(name, what):
    """What the gradient reads of the plan may not change; its dict may, as the call kept what it took."""
    t, call, plan = _calls()[name]
    leaf = t.clone().requires_grad_(True)
    out = call(leaf)
    out.backward(torch.ones_like(out))
    want = leaf.grad.clone()
    leaf.grad = None
    out = call(leaf)
    kept = plan[what]
    plan[what] = torch.zeros_like(kept)         # another tensor in the dict
    out.backward(torch.ones_like(out))
    assert torch.equal(leaf.grad, want)
    plan[what] = kept
    out = call(leaf)
    kept.add_(0)                                # the same tensor, written
    if what == "ids" and not name.startswith("lora"):
        out.backward(torch.ones_like(out))      # a tensor of its own, which this gradient does not read
    else:                                       # the others share memory, and so what torch counts
        with pytest.raises(RuntimeError, match="plan"):
            out.backward(torch.ones_like(out))
    out = call(leaf)                            # written before the call: what the call saw
    out.backward(torch.ones_like(out))


def test_a_plan_made_in_inference_mode_still_serves():
    ids = torch.randint(0, 3, (50,), device=DEV).to(torch.int32)
    with torch.inference_mode():
        plan = P.group_rows(ids, 3)
    x = torch.randn(50, 16, device=DEV, requires_grad=True)
    P.dispatch_rows(x, plan).sum().backward()
    assert torch.equal(x.grad, torch.ones_like(x))
