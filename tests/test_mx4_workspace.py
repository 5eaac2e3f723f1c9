"""Workspaces of the 4-bit FFN: what is sized for the largest batch has to hold every smaller one."""
import pytest
import torch

import paper_2606_15453_b200 as P
from datagen import stacks

DEV = "cuda:0"


@pytest.mark.parametrize("H,I", [(32, 32), (256, 160), (2048, 768), (2048, 2048), (4096, 14336)])
def test_scratch_for_a_batch_serves_every_smaller_one(H, I):
    """The partial sums take pairs * splits rows, and the splits fall from 8 to 4 behind 32 pairs and to 2 behind
    128: the size of 34 pairs has to cover the 8 x 32 rows of 32 pairs."""
    f = P.lib().stmoe_mx4_ffn_scratch_bytes
    for top_k in range(1, 33):
        sizes = [f(b, top_k, H, I) for b in range(1, 65)]
        assert sizes[0] > 0 and sizes == sorted(sizes)
    for batch in range(1, 65):
        sizes = [f(batch, k, H, I) for k in range(1, 33)]
        assert sizes == sorted(sizes)


def _stack(cfg, max_batch):
    st = P.Stack.from_config(cfg, max_batch=max_batch, dtype="mx4")
    router = stacks.router_weights(cfg)
    for l in range(cfg.n_layers):
        st.load_router(l, router[l])
        for shared, n in ((False, cfg.n_experts), (True, cfg.n_shared)):
            for e in range(n):
                w = stacks.expert_weights(cfg, l, e, shared, device=DEV)
                q = P.mx4_expert(w["gate"], w["up"], w["down"])
                torch.cuda.synchronize()
                st.load_experts(l, e, q["gate"], q["up"], q["down"], q["scales"], shared)
    return st


@pytest.mark.gpu
@pytest.mark.parametrize("E,K,shared,H,I,most,batches", [
    (8, 2, 0, 2048, 2048, 20, (16, 1)),       # 40 pairs sized, 32 used: six splits
    (16, 4, 0, 2048, 2048, 33, (27, 8)),      # 132 sized, 108 and 32 used
    (6, 2, 1, 256, 2080, 11, (10, 3)),        # with a shared expert: 33 sized, 30 used
])
def test_fewer_sequences_than_a_stack_has_room_for(E, K, shared, H, I, most, batches):
    """A step of fewer sequences has the bits that a stack sized for them has."""
    cfg = stacks.CONFIGS["C2"].scaled(n_layers=2, profile_tokens=0, n_experts=E, top_k=K, n_shared=shared, hidden=H, inter=I)
    wide = _stack(cfg, most)
    for B in batches:
        own = _stack(cfg, B)
        x = stacks.token_inputs(cfg, B, 2)[1].to(DEV)
        a, b, one = (torch.empty(B, H, device=DEV) for _ in range(3))
        torch.cuda.synchronize()
        wide.decode_token(x, a)
        own.decode_token(x, b)
        one.copy_(x)
        for l in range(cfg.n_layers):
            own.decode_step(l, one, one)
        torch.cuda.synchronize()
        assert torch.isfinite(a).all() and torch.equal(a, b) and torch.equal(a, one)
        own.stats(), own.close()
    wide.stats(), wide.close()


@pytest.mark.gpu
def test_scratch_sized_for_the_largest_batch_is_taken_for_smaller_ones():
    E, K, H, I = 8, 2, 256, 2080
    scratch = torch.empty(P.moe_ffn_scratch_bytes(17, K, H, I, "mx4"), dtype=torch.uint8, device=DEV)
    g = torch.Generator().manual_seed(1)
    images = torch.stack([P.mx4_expert(*(0.02 * torch.randn(*s, generator=g).to(DEV) for s in ((I, H), (I, H), (H, I))))["image"]
                          for _ in range(E)])
    h = torch.randn(17, H, generator=g).to(DEV)
    ids = torch.stack([torch.randperm(E, generator=g)[:K] for _ in range(17)]).to(torch.int32).to(DEV)
    w = torch.rand(17, K, generator=g).to(DEV)
    for b in (17, 16, 5, 1):
        own = torch.empty(P.moe_ffn_scratch_bytes(b, K, H, I, "mx4"), dtype=torch.uint8, device=DEV)
        got, want = (torch.empty(b, H, device=DEV) for _ in range(2))
        P.moe_ffn(h[:b], None, ids[:b], w[:b], images, "mx4", E, H, I, 0.1, got, scratch)
        P.moe_ffn(h[:b], None, ids[:b], w[:b], images, "mx4", E, H, I, 0.1, want, own)
        assert torch.isfinite(got).all() and torch.equal(got, want)
