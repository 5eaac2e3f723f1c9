"""Routed FFN over 4-bit expert images, stand-alone and inside stacks, against 64 bits."""
import numpy as np
import pytest
import torch

import mx4_reference as R
import paper_2606_15453_b200 as P
from datagen import stacks
from helpers import check_layer, rel_err
from oracle.stack import OracleStack

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _experts(g, E, H, I, sigma=0.02):
    """Images of E experts and their matrices as the images hold them (fp64)."""
    imgs, mats = [], []
    for _ in range(E):
        w = [sigma * torch.randn(*s, generator=g) for s in ((I, H), (I, H), (H, I))]
        q = P.mx4_expert(*[t.to(DEV) for t in w])
        imgs.append(q["image"])
        img = q["image"].cpu().numpy()
        nc, ns = H * I // 2, H * I // 32
        mats.append([R.values(img[i * nc:(i + 1) * nc].reshape(r, c // 2), img[3 * nc + i * ns:3 * nc + (i + 1) * ns].reshape(r, c // 32))
                     for i, (r, c) in enumerate(((I, H), (I, H), (H, I)))])
    return torch.stack(imgs), mats


def _problem(seed, B, E, K, H, I):
    g = torch.Generator().manual_seed(seed)
    img, mats = _experts(g, E, H, I)
    h = torch.randn(B, H, generator=g) * torch.exp(0.5 * torch.randn(B, 1, generator=g))
    h[:, ::37] *= 20
    inv = 1 / torch.sqrt((h.double() ** 2).mean(1) + 1e-6)
    z = torch.randn(B, E, generator=g)
    ids = torch.sort(z.topk(K, 1).indices, 1).values.to(torch.int32)
    w = torch.softmax(z, 1).gather(1, ids.long())
    return img, mats, h, inv.float(), ids, w


def _run(img, h, inv, ids, w, E, H, I, r=0.1, fn="ffn"):
    B, K = ids.shape
    out = torch.full((B, H), float("nan"), device=DEV)
    a = (h.to(DEV), None if inv is None else inv.to(DEV), ids.to(DEV), w.to(DEV), img, "mx4", E, H, I, r, out)
    if fn == "static":
        P.moe_ffn_static(*a)
    else:
        scratch = torch.full((P.moe_ffn_scratch_bytes(B, K, H, I, "mx4"),), 0xFF, dtype=torch.uint8, device=DEV)
        P.moe_ffn(*a, scratch)
    return out.cpu()


def _want_and_bound(mats, h, inv, ids, w, r=0.1):
    """fp64 result and what it may be off by: an activation is off by less than 2^-22 of the largest
    magnitude of its block of 32, a sum of n products by at most n 2^-23 of its magnitudes, SiLU * up by
    |SiLU'| <= 1.1 on top of 2^-19 of its value, and every store by 2^-24."""
    h, w = h.double().numpy(), w.double().numpy()
    inv = np.ones(len(h)) if inv is None else inv.double().numpy()
    out, tol = h.copy(), np.zeros_like(h)

    def linear(m, x, dx):
        block = np.repeat(np.abs(x).reshape(-1, 32).max(1), 32)
        a = np.abs(m)
        return m @ x, a @ (dx + 2.0 ** -22 * block) + (len(x) + 8) * 2.0 ** -23 * (a @ np.abs(x))

    for b in range(len(h)):
        x = h[b] * inv[b]
        for k, e in enumerate(ids[b].tolist()):
            if not 0 <= e < len(mats):
                continue
            g, dg = linear(mats[e][0], x, 2.0 ** -23 * np.abs(x))
            u, du = linear(mats[e][1], x, 2.0 ** -23 * np.abs(x))
            s = g / (1 + np.exp(-g))
            act = s * u
            y, dy = linear(mats[e][2], act, 1.1 * dg * np.abs(u) + (np.abs(s) + 1.1 * dg) * du + 2.0 ** -19 * np.abs(act))
            out[b] += r * w[b, k] * y
            tol[b] += abs(r * w[b, k]) * (dy + 2.0 ** -21 * np.abs(y))
        tol[b] += 2.0 ** -23 * np.abs(out[b])
    return out, tol


@pytest.mark.parametrize("B,E,K,H,I", [(1, 8, 2, 32, 32), (1, 16, 4, 256, 96), (3, 5, 2, 96, 160), (7, 1, 1, 64, 64), (13, 2, 1, 320, 224),
                                       (64, 3, 2, 128, 352), (64, 40, 6, 256, 128), (25, 9, 9, 1024, 288), (1, 6, 3, 2048, 1408), (30, 4, 2, 512, 2080)])
def test_ffn_against_64_bits(B, E, K, H, I):
    img, mats, h, inv, ids, w = _problem(B + E + H + I, B, E, K, H, I)
    want, tol = _want_and_bound(mats, h, inv, ids, w)
    got = _run(img, h, inv, ids, w, E, H, I).double().numpy()
    assert (np.abs(got - want) <= tol).all(), float((np.abs(got - want) / tol).max())
    want, tol = _want_and_bound(mats, h, None, ids, w)
    got = _run(img, h, None, ids, w, E, H, I).double().numpy()
    assert (np.abs(got - want) <= tol).all()


@pytest.mark.parametrize("scale", [1.0, 2.0 ** 60, 2.0 ** -60])
def test_ffn_exact_where_the_arithmetic_is(scale):
    """Eight ones in h against gate weights of 6: g = 48, where SiLU is the identity in fp32; the up sums are
    multiples of 1/2 up to 48, their products with 48 multiples of 24, the down sums multiples of 12
    below 2^20: nothing is rounded, on any path of the sums and planes."""
    H, I, E, B, K = 96, 192, 3, 9, 2
    g = torch.Generator().manual_seed(7)
    nc, ns = H * I // 2, H * I // 32
    img = torch.zeros(E, P.expert_image_bytes(H, I, "mx4"), dtype=torch.uint8)
    img[:, nc:3 * nc] = torch.randint(0, 256, (E, 2 * nc), generator=g, dtype=torch.uint8)
    img[:, :nc] = 0x77                                        # 6, 6
    img[:, 3 * nc:3 * nc + 3 * ns] = 127
    mats = [[R.values(img[e, i * nc:(i + 1) * nc].numpy().reshape(r, c // 2), np.full((r, c // 32), 127, np.uint8))
             for i, (r, c) in enumerate(((I, H), (I, H), (H, I)))] for e in range(E)]
    h = torch.zeros(B, H)
    for b in range(B):
        h[b, torch.randperm(H, generator=g)[:8]] = scale
    inv = torch.full((B,), 1 / scale)
    ids = torch.tensor([[b % 3, (b + 1) % 3] for b in range(B)], dtype=torch.int32)
    w = torch.tensor([[1.0, 0.5]] * B)
    got = _run(img.to(DEV), h, inv, ids, w, E, H, I, r=scale).double().numpy() / scale
    x = (h / scale).double().numpy()
    for b in range(B):
        y = x[b].copy()
        for k in range(K):
            m = mats[ids[b, k]]
            y += float(w[b, k]) * (m[2] @ ((m[0] @ x[b]) * (m[1] @ x[b])))
        assert (got[b] == y).all()


def test_ffn_same_bits_on_every_call_and_from_the_static_entry():
    img, _, h, inv, ids, w = _problem(3, 20, 6, 2, 512, 352)
    a = _run(img, h, inv, ids, w, 6, 512, 352)
    assert torch.isfinite(a).all()
    for fn in ("ffn", "static"):
        assert torch.equal(a, _run(img, h, inv, ids, w, 6, 512, 352, fn=fn))


def test_ffn_choices_without_an_expert_add_nothing():
    img, mats, h, inv, ids, w = _problem(4, 5, 4, 3, 128, 96)
    ids[0], ids[1, 0], ids[2, 1] = -1, 4, 1 << 30
    want, tol = _want_and_bound(mats, h, inv, ids, w)
    got = _run(img, h, inv, ids, w, 4, 128, 96)
    assert torch.equal(got[0], h[0])
    assert (np.abs(got.double().numpy() - want) <= tol).all()


def test_ffn_one_expert_twice_in_a_row():
    img, mats, h, inv, ids, w = _problem(5, 14, 3, 2, 64, 64)
    ids[:, 0] = ids[:, 1]
    want, tol = _want_and_bound(mats, h, inv, ids, w)
    assert (np.abs(_run(img, h, inv, ids, w, 3, 64, 64).double().numpy() - want) <= tol).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_ffn_non_finite_tokens_stay_alone(bad):
    img, _, h, inv, ids, w = _problem(6, 20, 3, 2, 128, 96)
    clean = _run(img, h, inv, ids, w, 3, 128, 96)
    h[7, 33] = bad
    got = _run(img, h, inv, ids, w, 3, 128, 96)
    rest = [b for b in range(20) if b != 7]
    assert got[7].isnan().any() and torch.equal(got[rest], clean[rest])


def test_ffn_tiny_and_huge_activations():
    img, mats, h, _, ids, w = _problem(8, 6, 3, 2, 64, 96)
    for s in (1e-30, 1e25):
        hs = h * s
        inv = 1 / torch.sqrt((hs.double() ** 2).mean(1)).float()
        want, tol = _want_and_bound(mats, hs, inv, ids, w, r=s)
        got = _run(img, hs, inv, ids, w, 3, 64, 96, r=s).double().numpy()
        assert (np.abs(got - want) <= tol).all()


def test_ffn_on_a_stream_and_replayed():
    img, _, h, inv, ids, w = _problem(9, 4, 6, 2, 256, 160)
    h, inv, ids, w = h.to(DEV), inv.to(DEV), ids.to(DEV), w.to(DEV)
    scratch = [torch.empty(P.moe_ffn_scratch_bytes(4, 2, 256, 160, "mx4"), dtype=torch.uint8, device=DEV) for _ in range(2)]
    want, out = torch.empty(4, 256, device=DEV), torch.empty(4, 256, device=DEV)
    P.moe_ffn(h, inv, ids, w, img, "mx4", 6, 256, 160, 0.1, want, scratch[0])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    P.moe_ffn(h, inv, ids, w, img, "mx4", 6, 256, 160, 0.1, out, scratch[1], stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.moe_ffn(h, inv, ids, w, img, "mx4", 6, 256, 160, 0.1, out, scratch[1])
    h.mul_(1.5)
    ids.copy_((ids + 1) % 6)
    graph.replay()
    P.moe_ffn(h, inv, ids, w, img, "mx4", 6, 256, 160, 0.1, want, scratch[0])
    assert torch.equal(out, want)


# ---- stacks ------------------------------------------------------------------------------------

def _stack_pair(cfg, B, **kw):
    """A stack with MX4 experts and the fp32 reference on the values that the images hold (they are
    bf16 numbers: one significant bit behind the first, an 8-bit exponent)."""
    router = stacks.router_weights(cfg)
    st = P.Stack.from_config(cfg, max_batch=B, dtype="mx4", **kw)
    cpu = {}
    for l in range(cfg.n_layers):
        st.load_router(l, router[l])
        for shared, n in ((False, cfg.n_experts), (True, cfg.n_shared)):
            for e in range(n):
                w = stacks.expert_weights(cfg, l, e, shared, device=DEV)
                q = P.mx4_expert(w["gate"], w["up"], w["down"])
                torch.cuda.synchronize()
                st.load_experts(l, e, q["gate"], q["up"], q["down"], q["scales"], shared)
                H, I = cfg.hidden, cfg.inter
                ns = H * I // 32
                cpu[l, e, shared] = {
                    k: torch.from_numpy(R.values(q[k].cpu().numpy(), q["scales"][i * ns:(i + 1) * ns].view(q[k].shape[0], -1).cpu().numpy())).to(torch.bfloat16)
                    for i, k in enumerate(("gate", "up", "down"))}
    return st, OracleStack(cfg, router, lambda l, e, s=False: cpu[l, e, s], batch=B, mode=kw.get("mode", "st"),
                           prefetch_limit=kw.get("prefetch_limit", 0))


@pytest.mark.parametrize("B,shared,slots", [(1, 0, 0), (1, 2, 0), (5, 1, 0), (40, 0, 0), (1, 0, 9), (4, 0, 12), (3, 2, 8)])
def test_stack_layer_by_layer(B, shared, slots):
    cfg = stacks.CONFIGS["C2"].scaled(n_layers=3, profile_tokens=2, hidden=256, inter=160, n_experts=12, top_k=2, n_shared=shared,
                                      cache_slots=max(slots, 2 * B) if slots else 0)
    st, orc = _stack_pair(cfg, B)
    tight = cfg.scaled(dtype="f32")           # the tolerance of fp32 stacks, 1e-4
    x = stacks.token_inputs(cfg, B, 4)
    K = cfg.top_k
    ids, w = torch.empty(B, K, dtype=torch.int32, device=DEV), torch.empty(B, K, device=DEV)
    pred, npred = torch.empty(B, st.max_pred, dtype=torch.int32, device=DEV), torch.empty(B, dtype=torch.int32, device=DEV)
    flags, out = torch.empty(B, dtype=torch.int32, device=DEV), torch.empty(B, cfg.hidden, device=DEV)
    for t in range(4):
        h = x[t].numpy()
        for l in range(cfg.n_layers):
            st.decode_step(l, torch.from_numpy(h).to(DEV), out, ids, w, pred, npred, flags)
            torch.cuda.synchronize()
            o = orc.layer_step(l, h)
            g = dict(h_out=out.cpu().numpy(), ids=ids.cpu().numpy(), w=w.cpu().numpy(), ties=flags.cpu().numpy() & 1)
            check_layer(tight, g, o, h, f"t={t} l={l}")
            if not (g["ids"] == o["ids"]).all():
                return                        # a near tie went the other way: the tables part here
            h = o["h_out"]
    assert st.stats()["decode_steps"] == 4
    st.close()


@pytest.mark.parametrize("B,slots", [(1, 0), (6, 0), (2, 9)])
def test_stack_whole_tokens_and_host_buffers(B, slots):
    cfg = stacks.CONFIGS["C2"].scaled(n_layers=3, profile_tokens=2, hidden=128, inter=96, n_experts=10, top_k=2, n_shared=0, cache_slots=slots)
    st, orc = _stack_pair(cfg, B)
    x = stacks.token_inputs(cfg, B, 5)
    out = torch.empty(B, cfg.hidden, device=DEV)
    ids = torch.empty(cfg.n_layers, B, cfg.top_k, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    for t in range(5):
        h_ref, per = orc.decode_token(x[t].numpy())
        if t == 4:
            got, gids = torch.empty(B, cfg.hidden), torch.empty(cfg.n_layers, B, cfg.top_k, dtype=torch.int32)
            st.decode_token_host(x[t].contiguous(), got, gids)
        else:
            xd = x[t].to(DEV)
            torch.cuda.synchronize()
            st.decode_token(xd, out, ids, stream=side)      # captured and replayed where the stack is resident
            torch.cuda.synchronize()
            got, gids = out.cpu(), ids.cpu()
        if any((gids[l].numpy() != per[l]["ids"]).any() for l in range(cfg.n_layers)):
            assert sum(int(r["ties"].sum()) for r in per) > 0
            break
        assert rel_err(got.numpy(), h_ref) <= 1e-4
    st.stats()
    st.close()


@pytest.mark.parametrize("B", [1, 7, 33])
def test_stack_replayed_steps_have_the_bits_of_single_layers(B):
    """Many layers whose launches overlap and share the work list's and the planes' buffers, against
    the same layers one at a time with a synchronisation behind each."""
    cfg = stacks.CONFIGS["C2"].scaled(n_layers=10, profile_tokens=0, hidden=192, inter=160, n_experts=20, top_k=3, n_shared=1)
    a, _ = _stack_pair(cfg, B)
    b, _ = _stack_pair(cfg, B)
    x = stacks.token_inputs(cfg, B, 12)
    side = torch.cuda.Stream()
    h, out, one = (torch.empty(B, cfg.hidden, device=DEV) for _ in range(3))
    for t in range(12):
        h.copy_(x[t])
        torch.cuda.synchronize()
        a.decode_token(h, out, stream=side)
        side.synchronize()
        one.copy_(h)
        for l in range(cfg.n_layers):
            b.decode_step(l, one, one)
            torch.cuda.synchronize()
        assert torch.equal(out, one), t
    a.close(), b.close()


def test_stack_kernel_timing_covers_the_projections():
    cfg = stacks.CONFIGS["C2"].scaled(n_layers=2, profile_tokens=0, hidden=128, inter=96, n_experts=8, top_k=2, n_shared=0)
    st, _ = _stack_pair(cfg, 2)
    st.set_kernel_timing(True)
    x = stacks.token_inputs(cfg, 2, 1)[0].to(DEV)
    st.decode_token(x, torch.empty_like(x))
    s = st.stats()
    assert s["timed_ffn_launches"] == 2 and s["gate_up_ms"] > 0 and s["down_ms"] > 0
    st.close()


def test_a_run_of_them_together():
    """Prefill through a layer of 4-bit experts as a program would write it: the router's counts group the
    tokens, their losses come with them, and the experts' products run on quantised activations."""
    T, E, K, H, I = 300, 8, 2, 256, 160
    g = torch.Generator().manual_seed(31)
    img, mats = _experts(g, E, H, I)
    nc, ns = H * I // 2, H * I // 32

    def matrices(i, r, c):
        return (img[:, i * nc:(i + 1) * nc].reshape(E, r, c // 2).contiguous(),
                img[:, 3 * nc + i * ns:3 * nc + (i + 1) * ns].reshape(E, r, c // 32).contiguous())
    h = torch.randn(T, H, generator=g).to(DEV)
    logits = torch.randn(T, E, generator=g).to(DEV)
    ids = logits.topk(K, 1).indices.to(torch.int32)
    f = P.router_balance(logits, ids)
    d = P.router_balance_backward(logits, f, torch.tensor([1.0, 0.1], device=DEV))
    order = torch.argsort(ids.flatten(), stable=True)
    tok = order // K
    x = P.mx4_quantize(h.index_select(0, tok))
    gate = P.mx4_matmul(x, matrices(0, I, H), counts=f["counts"], dtype=torch.float32)
    up = P.mx4_matmul(x, matrices(1, I, H), counts=f["counts"], dtype=torch.float32)
    a = P.mx4_quantize(torch.nn.functional.silu(gate) * up)
    y = P.mx4_matmul(a, matrices(2, H, I), counts=f["counts"], dtype=torch.float32)
    assert d.isfinite().all() and f["counts"].sum().item() == T * K
    xv = R.values(*[t.cpu().numpy() for t in x])
    av = R.values(*[t.cpu().numpy() for t in a])
    e = ids.flatten()[order].cpu().numpy()
    for i in range(0, T * K, 7):
        for got, m, v in ((gate, 0, xv), (up, 1, xv), (y, 2, av)):
            w = mats[e[i]][m]
            tol = w.shape[1] * 2.0 ** -23 * (np.abs(w) @ np.abs(v[i]))
            assert (np.abs(got[i].double().cpu().numpy() - w @ v[i]) <= tol).all()
