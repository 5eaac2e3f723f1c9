"""The 4-bit FFN at the sizes of the repository's large experts (4096 x 14336: 16 reduction stages up, 56 down, both
split), against 64 bits on the device."""
import pytest
import torch

import paper_2606_15453_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _values(codes, scales, rows, cols):
    """fp64 [rows][cols] of codes and scale bytes, by the format's definition."""
    half = torch.stack([codes & 15, codes >> 4], -1).view(rows, cols).long()
    v = torch.tensor(LEVELS + [-x for x in LEVELS], dtype=torch.float64, device=DEV)[half]
    return v * torch.exp2(scales.view(rows, cols // 32).double() - 127).repeat_interleave(32, 1)


def _linear(m, x, dx):
    """m @ x and what the kernel's may be off by: an activation by less than 2^-22 of the largest magnitude of its
    32, a sum of n products by n 2^-23 of its magnitudes (see the small sizes' test)."""
    block = x.abs().view(-1, 32).amax(1).repeat_interleave(32)
    a = m.abs()
    return m @ x, a @ (dx + 2.0 ** -22 * block) + (len(x) + 8) * 2.0 ** -23 * (a @ x.abs())


@pytest.mark.parametrize("B,E,K,H,I", [(1, 3, 2, 4096, 14336), (4, 2, 2, 4096, 14336), (16, 2, 1, 4096, 14336), (33, 5, 3, 4096, 1536)])
def test_large_experts_against_64_bits(B, E, K, H, I):
    g = torch.Generator(device=DEV).manual_seed(B + I)
    images = torch.stack([P.mx4_expert(*(0.02 * torch.randn(*s, generator=g, device=DEV) for s in ((I, H), (I, H), (H, I))))["image"]
                          for _ in range(E)])
    h = torch.randn(B, H, generator=g, device=DEV)
    h[:, ::37] *= 20
    inv = torch.rsqrt((h * h).mean(1) + 1e-6)
    z = torch.randn(B, E, generator=g, device=DEV)
    ids = z.topk(K, 1).indices.to(torch.int32)
    w = torch.softmax(z, 1).gather(1, ids.long())
    out = torch.full((B, H), float("nan"), device=DEV)
    scratch = torch.full((P.moe_ffn_scratch_bytes(B, K, H, I, "mx4"),), 0xFF, dtype=torch.uint8, device=DEV)
    P.moe_ffn(h, inv, ids, w, images, "mx4", E, H, I, 0.1, out, scratch)
    torch.cuda.synchronize()
    want, tol = h.double(), torch.zeros(B, H, dtype=torch.float64, device=DEV)
    nc, ns = H * I // 2, H * I // 32
    for e in range(E):
        rows = (ids == e).nonzero().tolist()
        if not rows:
            continue
        img = images[e]
        mats = [_values(img[i * nc:(i + 1) * nc], img[3 * nc + i * ns:3 * nc + (i + 1) * ns], r, c)
                for i, (r, c) in enumerate(((I, H), (I, H), (H, I)))]
        for b, k in rows:
            x = h[b].double() * inv[b].double()
            gate, dg = _linear(mats[0], x, 2.0 ** -23 * x.abs())
            up, du = _linear(mats[1], x, 2.0 ** -23 * x.abs())
            s = gate * torch.sigmoid(gate)
            act = s * up
            y, dy = _linear(mats[2], act, 1.1 * dg * up.abs() + (s.abs() + 1.1 * dg) * du + 2.0 ** -19 * act.abs())
            share = 0.1 * w[b, k].double()
            want[b] += share * y
            tol[b] += share * (dy + 2.0 ** -21 * y.abs())
    tol += 2.0 ** -23 * want.abs()
    assert ((out.double() - want).abs() <= tol).all()
    # the bound is of the worst case; what the error comes to as a whole is far smaller
    assert float((out.double() - want).norm() / want.norm()) <= 2.0 ** -21
