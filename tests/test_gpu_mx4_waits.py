"""Bounded waits of the MX4 kernels that run out, by a lowered poll limit (no barrier is broken: the limit
alone ends the waits): the kernels end, what depends on an expired wait is NaN, the rest is as it should be, and the
next call with the default limit is whole."""
import pytest
import torch

import paper_2606_15453_b200 as P
from paper_2606_15453_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DEFAULT = 1 << 22


@pytest.fixture
def polls():
    yield binding.mx4_poll_limit
    torch.cuda.synchronize()
    binding.mx4_poll_limit(DEFAULT)


def _rows(g, rows, nb):
    return (torch.randint(0, 256, (rows, nb * 16), generator=g, device=DEV, dtype=torch.uint8),
            torch.randint(126, 129, (rows, nb), generator=g, device=DEV, dtype=torch.uint8))


def _product(seed, counts, behind, n, nb, dt, pad):
    g = torch.Generator(device=DEV).manual_seed(seed)
    E, m = len(counts), sum(counts) + behind
    bc, bs = _rows(g, E * n, nb)
    a, b = _rows(g, m, nb), (bc.view(E, n, -1), bs.view(E, n, -1))
    cd = torch.tensor(counts, dtype=torch.int32, device=DEV)
    out = torch.full((m, n + pad), 7.0, dtype=dt, device=DEV)[:, :n]

    def call():
        out.fill_(7.0)
        flags = torch.zeros(1, dtype=torch.int32, device=DEV)
        P.mx4_matmul(a, b, counts=cd, out=out, flags=flags)
        torch.cuda.synchronize()
        return out.clone(), flags.item()
    return call, sum(counts)


# a tile or more for every CTA, whole lines of the output and not; a reduction split over clusters; groups
PRODUCTS = [([700], 0, 40000, 9, torch.bfloat16, 0), ([700], 3, 40001, 9, torch.float32, 0), ([300, 0, 41], 5, 20000, 12, torch.float16, 8),
            ([5], 2, 512, 64, torch.bfloat16, 0), ([3, 4], 0, 200, 24, torch.float32, 1)]


@pytest.mark.parametrize("case", range(len(PRODUCTS)))
def test_product_whose_waits_give_up_at_once_is_nan_throughout(polls, case):
    call, used = _product(case, *PRODUCTS[case])
    want, flag = call()
    assert flag == 0 and want[:used].isfinite().all()
    polls(0)
    got, flag = call()
    assert flag == 1 and got[:used].isnan().all() and (got[used:] == 7).all()
    polls(DEFAULT)
    again, flag = call()
    assert flag == 0 and torch.equal(again, want)


@pytest.mark.parametrize("limit", [1, 2, 4, 8])
@pytest.mark.parametrize("case", range(len(PRODUCTS)))
def test_product_whose_waits_give_up_on_the_way_is_whole_or_nan(polls, case, limit):
    """A few polls, some microseconds each: some waits hold and some run out, with loads and MMAs under way."""
    call, used = _product(case, *PRODUCTS[case])
    want, _ = call()
    polls(limit)
    for _ in range(3):
        got, flag = call()
        bad = got[:used].isnan()
        assert torch.equal(got[:used][~bad], want[:used][~bad]) and (got[used:] == 7).all()
        assert flag == 1 or not bad.any()
    polls(DEFAULT)
    again, flag = call()
    assert flag == 0 and torch.equal(again, want)


def _ffn(B, E, K, H, I, static=False):
    g = torch.Generator(device=DEV).manual_seed(B + E + H)
    images = torch.stack([P.mx4_expert(*(0.02 * torch.randn(*s, generator=g, device=DEV) for s in ((I, H), (I, H), (H, I))))["image"]
                          for _ in range(E)])
    h = torch.randn(B, H, generator=g, device=DEV)
    ids = torch.stack([torch.randperm(E, generator=g, device=DEV)[:K] for _ in range(B)]).to(torch.int32)
    w = torch.rand(B, K, generator=g, device=DEV) + 0.1
    scratch = torch.empty(P.moe_ffn_scratch_bytes(B, K, H, I, "mx4"), dtype=torch.uint8, device=DEV)
    ids[-1] = -1                              # a sequence without experts depends on nothing

    def call():
        out = torch.full((B, H), 7.0, device=DEV)
        a = (h, None, ids, w, images, "mx4", E, H, I, 0.1, out)
        P.moe_ffn_static(*a) if static else P.moe_ffn(*a, scratch)
        torch.cuda.synchronize()
        return out
    return call, h


# gate/up's reduction split over clusters; tasks beyond the CTAs in both projections; the static entry
FFNS = [(2, 4, 1, 2048, 256, False), (20, 24, 6, 1024, 1408, False), (64, 8, 2, 2048, 2080, False), (3, 6, 2, 512, 352, True)]


@pytest.mark.parametrize("case", range(len(FFNS)))
def test_ffn_whose_waits_give_up_at_once_is_nan_throughout(polls, case):
    """The scratch still holds the activations and partial sums of the call before: none of them may be taken."""
    call, h = _ffn(*FFNS[case])
    want = call()
    assert want.isfinite().all()
    polls(0)
    got = call()
    assert got[:-1].isnan().all() and torch.equal(got[-1], h[-1])
    polls(DEFAULT)
    assert torch.equal(call(), want)


@pytest.mark.parametrize("limit", [1, 2, 4, 8])
@pytest.mark.parametrize("case", range(len(FFNS)))
def test_ffn_whose_waits_give_up_on_the_way_is_whole_or_nan(polls, case, limit):
    call, h = _ffn(*FFNS[case])
    want = call()
    polls(limit)
    for _ in range(3):
        got = call()
        bad = got.isnan()
        assert torch.equal(got[~bad], want[~bad]) and torch.equal(got[-1], h[-1])
    polls(DEFAULT)
    assert torch.equal(call(), want)


def test_stack_whose_waits_give_up_reports_a_timeout(polls):
    from datagen import stacks
    cfg = stacks.CONFIGS["C2"].scaled(n_layers=2, profile_tokens=0, hidden=256, inter=160, n_experts=8, top_k=2, n_shared=1)
    st = P.Stack.from_config(cfg, max_batch=3, dtype="mx4")
    router = stacks.router_weights(cfg)
    for l in range(cfg.n_layers):
        st.load_router(l, router[l])
        for shared, n in ((False, cfg.n_experts), (True, cfg.n_shared)):
            for e in range(n):
                w = stacks.expert_weights(cfg, l, e, shared, device=DEV)
                q = P.mx4_expert(w["gate"], w["up"], w["down"])
                torch.cuda.synchronize()
                st.load_experts(l, e, q["gate"], q["up"], q["down"], q["scales"], shared)
    x = stacks.token_inputs(cfg, 3, 1)[0].to(DEV)
    out = torch.full_like(x, 7.0)
    st.decode_step(0, x, out)
    torch.cuda.synchronize()
    assert out.isfinite().all()
    polls(0)
    st.decode_step(1, out, out)
    torch.cuda.synchronize()
    assert out.isnan().all()
    with pytest.raises(P.StmoeError, match="timed out"):
        st.stats()
    st.close()
