"""Cases of the MX4 and router-statistics operators: inputs, plain forms in elementary torch
operations, the library's calls, and the definitions in 64 bits.

Four kinds of case (`op`):
  roundtrip  rows quantised to MX4 (32-element blocks of e2m1 codes under one e8m0 scale) and read back
  product    activations quantised to MX4, times MX4 weights; rows sorted by expert with device counts
  ffn        routed SwiGLU FFN of a decode step over 4-bit expert images
  balance    router balance loss, z loss, per-expert counts and the gradient of the logits
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one token's hidden state on its way into a 4-bit product: latency
        dict(name="roundtrip_token", op="roundtrip", rows=1, cols=2048, pad=0, dtype="f32"),
        # the gate matrix of a large expert when a checkpoint is converted
        dict(name="roundtrip_expert", op="roundtrip", rows=14336, cols=4096, pad=0, dtype="bf16"),
        # a slice of a wider activation buffer whose width is no multiple of the block
        dict(name="roundtrip_ragged", op="roundtrip", rows=4099, cols=1413, pad=11, dtype="f16"),
        # gate and up projections of one expert for a handful of tokens
        dict(name="product_few", op="product", tokens=5, n=2816, k=2048, experts=1, dtype="bf16"),
        # prefill of a fine-grained MoE layer: 512 tokens, top-6 of 64 experts, uneven groups
        dict(name="product_experts", op="product", tokens=3077, n=2816, k=2048, experts=64, dtype="bf16"),
        # sizes that are multiples of nothing, a group now and then empty
        dict(name="product_odd", op="product", tokens=333, n=1001, k=1120, experts=5, dtype="f16"),
        # a long prefill through a large expert
        dict(name="product_long", op="product", tokens=8192, n=14336, k=4096, experts=1, dtype="bf16"),
        # one sequence through a layer of small experts
        dict(name="ffn_one", op="ffn", batch=1, experts=128, top_k=8, hidden=2048, inter=768),
        # a full batch: every expert is read, some by many tokens
        dict(name="ffn_batch", op="ffn", batch=64, experts=64, top_k=6, hidden=2048, inter=1408),
        # a few sequences through large experts
        dict(name="ffn_large", op="ffn", batch=4, experts=8, top_k=2, hidden=4096, inter=14336),
        # the routing of one short micro-batch
        dict(name="balance_short", op="balance", tokens=61, experts=64, top_k=6, dtype="f32"),
        # the routing of a whole training batch
        dict(name="balance_long", op="balance", tokens=524288, experts=128, top_k=8, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["roundtrip", "product", "ffn", "balance"])
    if op == "roundtrip":
        cols = _log(rng, 1, 14336)
        rows = _log(rng, 1, max(1, min(50000, (14336 * 4096) // cols)))
        return dict(op=op, rows=rows, cols=cols, pad=rng.choice([0, 0, 1, 8, 37]), dtype=rng.choice(["f32", "bf16", "f16"]))
    if op == "product":
        n, k = _log(rng, 16, 8192), 32 * _log(rng, 1, 128)
        experts = rng.choice([1, 1, 2, 8, 60])
        if experts * n * k > 1 << 30:
            experts = 1
        return dict(op=op, tokens=_log(rng, 1, 6000), n=n, k=k, experts=experts, dtype=rng.choice(["bf16", "f16"]))
    if op == "ffn":
        hidden, inter = 32 * _log(rng, 2, 128), 32 * _log(rng, 2, 128)
        experts = _log(rng, 1, 128)
        while experts * hidden * inter > 400_000_000:
            experts = (experts + 1) // 2
        return dict(op=op, batch=_log(rng, 1, 64), experts=experts, top_k=min(experts, _log(rng, 1, 8)), hidden=hidden, inter=inter)
    experts = _log(rng, 2, 256)
    return dict(op=op, tokens=_log(rng, 1, 200000), experts=experts, top_k=min(experts, _log(rng, 1, 8)), dtype=rng.choice(["f32", "bf16"]))


# ---- plain MX4 -------------------------------------------------------------------------------

def _blocks(x):
    """[R][C] -> fp32 [R][ceil(C/32)][32], zeros behind the last column."""
    rows, cols = x.shape
    nb = (cols + 31) // 32
    y = torch.zeros(rows, nb * 32, dtype=torch.float32, device=x.device)
    y[:, :cols] = x
    return y.view(rows, nb, 32)


def _pow2(e):
    """2^e in fp32 for integers -127..127, built from its bits (library powers may round)."""
    e = e.to(torch.int32)
    return torch.where(e > -127, (e + 127) << 23, torch.full_like(e, 1 << 22)).view(torch.float32)


def _plain_quantize(x):
    """Codes as numbers 0..15 [R][nb][32] and scale bytes [R][nb]."""
    v = _blocks(x)
    a = v.abs()
    amax = a.amax(2)
    e = (torch.frexp(amax).exponent - 3).clamp(-127, 127)      # floor(log2(amax)) - 2
    e = torch.where(amax == 0, torch.full_like(e, -127), e)
    bad = ~torch.isfinite(amax)                                # amax is NaN where any value is
    e = torch.where(bad, torch.zeros_like(e), e)
    a = a * _pow2(-e)[:, :, None]
    mag = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5))
    code = mag + 8 * torch.signbit(v).to(torch.uint8)
    byte = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return code, byte


def _pack(code, byte):
    rows, nb, _ = code.shape
    return (code[..., 0::2] | (code[..., 1::2] << 4)).reshape(rows, nb * 16), byte


def _value_pairs(device):
    m = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    m = torch.tensor(m + [-v for v in m], dtype=torch.float32, device=device)
    b = torch.arange(256, device=device)
    return torch.stack([m[b & 15], m[b >> 4]], 1)


def _plain_dequantize(codes, byte):
    """fp32 [R][nb*32] from packed codes [R][nb*16] and scale bytes [R][nb]."""
    rows, nb = byte.shape
    v = _value_pairs(codes.device).index_select(0, codes.reshape(-1).to(torch.int32)).view(rows, nb, 32)
    e = byte.to(torch.int32) - 127
    y = v * _pow2(torch.where(byte == 255, torch.zeros_like(e), e))[:, :, None]
    return torch.where((byte == 255)[:, :, None], torch.full_like(y, math.nan), y).view(rows, nb * 32)


# ---- inputs ----------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 2654435761 % (1 << 62))


def _activations(g, rows, cols, pad=0, dtype=torch.float32):
    """Normal values with a few loud channels and a few quiet rows, as hidden states have them;
    `pad` more columns in the buffer than in the view."""
    x = torch.randn(rows, cols + pad, generator=g, device="cuda")
    loud = torch.rand(cols + pad, generator=g, device="cuda") < 0.01
    x = torch.where(loud, x * 20, x) * torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    return x.to(dtype)[:, :cols]


def _weights(g, rows, cols):
    """MX4 codes and scales of N(0, 0.02) weights, a slice of rows at a time."""
    codes = torch.empty(rows, cols // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(rows, cols // 32, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 27) // cols)
    for r in range(0, rows, step):
        w = 0.02 * torch.randn(min(step, rows - r), cols, generator=g, device="cuda")
        codes[r:r + step], scales[r:r + step] = _pack(*_plain_quantize(w))
    return codes, scales


def _image_bytes(hidden, inter):
    return -(-(51 * hidden * inter // 32) // 256) * 256


def prepare(case, seed):
    g = _gen(seed)
    op = case["op"]
    s = dict(case)
    if op == "roundtrip":
        s["x"] = _activations(g, case["rows"], case["cols"], case["pad"], DTYPES[case["dtype"]])
        if case["rows"] > 3:
            s["x"][case["rows"] // 2] = 0      # a padding token
    elif op == "product":
        m, n, k, E = case["tokens"], case["n"], case["k"], case["experts"]
        s["x"] = _activations(g, m, k, 0, DTYPES[case["dtype"]])
        codes, scales = _weights(g, E * n, k)
        s["codes"], s["scales"] = codes.view(E, n, k // 2), scales.view(E, n, k // 32)
        if E == 1:
            s["counts"], s["most"] = None, m
        else:                                   # popularity of the experts falls off, some get nothing
            share = torch.rand(E, generator=g, device="cuda") ** 2 + 1e-3
            pick = torch.multinomial(share, m, replacement=True, generator=g)
            s["counts"] = torch.bincount(pick, minlength=E).to(torch.int32)
            s["most"] = int(s["counts"].max())
    elif op == "ffn":
        B, E, K, H, I = (case[n] for n in ("batch", "experts", "top_k", "hidden", "inter"))
        s["h"] = _activations(g, B, H)
        s["inv_rms"] = torch.rsqrt((s["h"] * s["h"]).mean(1) + 1e-6)
        img = torch.zeros(E, _image_bytes(H, I), dtype=torch.uint8, device="cuda")
        codes, scales = H * I // 2, H * I // 32
        for e in range(E):
            for i, (r, c) in enumerate(((I, H), (I, H), (H, I))):
                q = _weights(g, r, c)
                img[e, i * codes:(i + 1) * codes] = q[0].view(-1)
                img[e, 3 * codes + i * scales:3 * codes + (i + 1) * scales] = q[1].view(-1)
        s["images"] = img
        z = torch.randn(B, E, generator=g, device="cuda")
        s["ids"] = z.topk(K, 1).indices.sort(1).values.to(torch.int32)
        s["w"] = torch.softmax(z, 1).gather(1, s["ids"].long()).contiguous()
        s["h_out"] = torch.empty_like(s["h"])
        # a generous workspace, allocated once as a serving loop would
        s["scratch"] = torch.empty((4 << 20) + 8 * B * K * (I + 8 * H), dtype=torch.uint8, device="cuda")
    else:
        T, E, K = case["tokens"], case["experts"], case["top_k"]
        z = 2 * torch.randn(T, E, generator=g, device="cuda") + torch.randn(E, generator=g, device="cuda")
        z = z.to(DTYPES[case["dtype"]])
        mask = torch.rand(T, generator=g, device="cuda") < 0.9
        mask[0] = True
        ids = z.float().topk(K, 1).indices.sort(1).values.to(torch.int32)
        drop = torch.rand(T, generator=g, device="cuda") < 0.02
        ids[:, 0] = torch.where(drop, torch.full_like(ids[:, 0], -1), ids[:, 0])   # over capacity: not counted
        ids[~mask] = -1
        z[~mask] = torch.where(drop[~mask][:, None], torch.full_like(z[~mask], math.nan), z[~mask])  # padding holds anything
        s["logits"], s["ids"], s["mask"] = z.contiguous(), ids.contiguous(), mask
        s["grad"] = torch.tensor([0.01, 0.001], device="cuda") * (1 + torch.rand(2, generator=g, device="cuda"))
    return s


# ---- one pass --------------------------------------------------------------------------------

def run(s):
    op = s["op"]
    if own:
        import paper_2606_15453_b200 as P
        if op == "roundtrip":
            codes, scales = P.mx4_quantize(s["x"])
            return P.mx4_dequantize(codes, scales, s["cols"], dtype=s["x"].dtype)
        if op == "product":
            a = P.mx4_quantize(s["x"])
            return P.mx4_matmul(a, (s["codes"], s["scales"]), counts=s["counts"], dtype=s["x"].dtype)
        if op == "ffn":
            return P.moe_ffn(s["h"], s["inv_rms"], s["ids"], s["w"], s["images"], "mx4", s["experts"], s["hidden"],
                             s["inter"], 0.1, s["h_out"], s["scratch"])
        f = P.router_balance(s["logits"], s["ids"], mask=s["mask"])
        d = P.router_balance_backward(s["logits"], f, s["grad"], mask=s["mask"])
        return {"loss": f["loss"], "counts": f["counts"], "dlogits": d}
    return {"roundtrip": _plain_roundtrip, "product": _plain_product, "ffn": _plain_ffn, "balance": _plain_balance}[op](s)


def _plain_roundtrip(s):
    return _plain_dequantize(*_pack(*_plain_quantize(s["x"])))[:, :s["cols"]].to(s["x"].dtype).contiguous()


def _plain_product(s):
    x = _plain_dequantize(*_pack(*_plain_quantize(s["x"])))
    E, n, nb = s["scales"].shape
    w = _plain_dequantize(s["codes"].reshape(E * n, nb * 16), s["scales"].reshape(E * n, nb)).view(E, n, nb * 32)
    if s["counts"] is None:
        return torch.matmul(x, w[0].t()).to(s["x"].dtype)
    ends = torch.cumsum(s["counts"], 0)
    row = torch.arange(s["tokens"], device=x.device)
    e = torch.searchsorted(ends, row, right=True)
    at = row - (ends - s["counts"])[e]
    wide = torch.zeros(E, s["most"], nb * 32, device=x.device)
    wide[e, at] = x
    return torch.bmm(wide, w.transpose(1, 2))[e, at].to(s["x"].dtype)


def _plain_ffn(s):
    B, E, K, H, I = (s[n] for n in ("batch", "experts", "top_k", "hidden", "inter"))
    dense = B * K >= E                       # every expert once, or only the routed ones, a copy for each pair
    img = s["images"] if dense else s["images"][s["ids"].reshape(-1).long()]
    n, nc, ns = img.shape[0], H * I // 2, H * I // 32
    q = img[:, :3 * (nc + ns)].contiguous()
    codes, scales = q[:, :3 * nc].reshape(n, 3, nc), q[:, 3 * nc:].reshape(n, 3, ns)
    W = _plain_dequantize(codes.reshape(-1, 16), scales.reshape(-1, 1)).view(n, 3, H * I)
    gate, up, down = W[:, 0].view(n, I, H), W[:, 1].view(n, I, H), W[:, 2].view(n, H, I)
    x = s["h"] * s["inv_rms"][:, None]
    if dense:
        xs = x.t().expand(n, H, B)
    else:
        xs = x.repeat_interleave(K, 0).unsqueeze(2)
    a, u = torch.bmm(gate, xs), torch.bmm(up, xs)
    y = torch.bmm(down, a / (1 + torch.exp(-a)) * u)              # [n][H][B] or [pairs][H][1]
    if dense:
        share = torch.zeros(B, E, device=x.device).scatter_add(1, s["ids"].long(), s["w"])
        y = (y.permute(2, 0, 1) * share[:, :, None]).sum(1)
    else:
        y = (y.view(B, K, H) * s["w"][:, :, None]).sum(1)
    return s["h"] + 0.1 * y


def _plain_balance(s):
    E, K = s["experts"], s["top_k"]
    z = s["logits"].float()
    keep = s["mask"] & (z != -math.inf).any(1)
    z = torch.where(keep[:, None], z, torch.zeros_like(z))
    n = keep.sum().double().clamp(min=1)
    m = z.amax(1, keepdim=True)
    ex = torch.exp(z - m)
    tot = ex.sum(1, keepdim=True)
    p = ex / tot * keep[:, None]
    lse = torch.where(keep, m[:, 0] + torch.log(tot[:, 0]), torch.zeros_like(tot[:, 0]))
    ids = torch.where(keep[:, None] & (s["ids"] >= 0) & (s["ids"] < E), s["ids"], torch.full_like(s["ids"], E))
    counts = torch.zeros(E + 1, dtype=torch.int64, device=z.device).scatter_add(0, ids.reshape(-1).long(), torch.ones_like(ids.reshape(-1), dtype=torch.int64))[:E]
    f = counts.double() / (n * K)
    balance = E * (f * (p.sum(0, dtype=torch.float64) / n)).sum()
    zloss = (lse * lse).sum(dtype=torch.float64) / n
    f, n = f.float(), n.float()
    d = s["grad"][0] * E / n * p * (f - (p * f).sum(1, keepdim=True)) + s["grad"][1] * 2 / n * lse[:, None] * p
    return {"loss": torch.stack([balance, zloss]).float(), "counts": counts.to(torch.int32), "dlogits": d.to(s["logits"].dtype)}


# ---- what a pass cannot do without ------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "roundtrip":
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * n * SIZE[case["dtype"]] + 17 * case["rows"] * -(-case["cols"] // 32), "flops": 4 * n}
    if op == "product":
        m, n, k, E = case["tokens"], case["n"], case["k"], case["experts"]
        used = E if E == 1 else E * (1 - (1 - 1 / E) ** m)
        return {"bytes": int(m * k * SIZE[case["dtype"]] + used * n * k * 17 / 32 + m * n * SIZE[case["dtype"]]), "flops": 2 * m * n * k}
    if op == "ffn":
        B, E, K, H, I = (case[n] for n in ("batch", "experts", "top_k", "hidden", "inter"))
        used = E * (1 - (1 - K / E) ** B)
        return {"bytes": int(used * 51 * H * I / 32 + 8 * B * H), "flops": 6 * B * K * H * I}
    T, E, K = case["tokens"], case["experts"], case["top_k"]
    return {"bytes": T * (2 * E * SIZE[case["dtype"]] + 4 * K + 1), "flops": 16 * T * E}


# ---- the definitions in 64 bits ----------------------------------------------------------------

_LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _exact_rounded(x):
    """The values that the MX4 form of x stands for, in 64 bits: the nearest level, ties to the even code."""
    rows, cols = x.shape
    nb = -(-cols // 32)
    v = torch.nn.functional.pad(x.double(), (0, nb * 32 - cols)).view(rows * nb, 32)
    top = v.abs().max(1, keepdim=True).values
    power = ((top.contiguous().view(torch.int64) >> 52) - 1023).clamp(min=-125)    # floor(log2(top))
    step = ((power - 2 + 1023) << 52).view(torch.float64)
    level = torch.tensor(_LEVELS, dtype=torch.float64, device=x.device)
    mid = (level[1:] + level[:-1]) / 2
    a = (v.abs() / step).contiguous()
    lo, hi = torch.searchsorted(mid, a), torch.searchsorted(mid, a, right=True)
    pick = torch.where((lo == hi) | (lo % 2 == 0), lo, hi)
    return (torch.sign(v) * level[pick] * step).view(rows, nb * 32)[:, :cols]


def _exact_weights(codes, scales):
    """fp64 [..., k] from packed codes and scale bytes."""
    half = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    level = torch.tensor(_LEVELS + [-v for v in _LEVELS], dtype=torch.float64, device=codes.device)
    return level[half] * ((scales.long() - 127 + 1023) << 52).view(torch.float64).repeat_interleave(32, -1)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "roundtrip":
        return _exact_rounded(s["x"])
    if op == "product":
        x = _exact_rounded(s["x"])
        E = case["experts"]
        out = torch.empty(case["tokens"], case["n"], dtype=torch.float64, device="cuda")
        counts = [case["tokens"]] if s["counts"] is None else s["counts"].tolist()
        at = 0
        for e in range(E):
            w = _exact_weights(s["codes"][e], s["scales"][e])
            out[at:at + counts[e]] = x[at:at + counts[e]] @ w.T
            at += counts[e]
        return out
    if op == "ffn":
        B, K, H, I = (case[n] for n in ("batch", "top_k", "hidden", "inter"))
        nc, ns = H * I // 2, H * I // 32
        x = s["h"].double() * s["inv_rms"].double()[:, None]
        out = s["h"].double()
        ids = s["ids"].cpu().numpy()
        for e in np.unique(ids):
            b, k = (torch.from_numpy(i).cuda() for i in np.nonzero(ids == e))
            img = s["images"][int(e)]
            m = [_exact_weights(img[i * nc:(i + 1) * nc].view(r, c // 2), img[3 * nc + i * ns:3 * nc + (i + 1) * ns].view(r, c // 32))
                 for i, (r, c) in enumerate(((I, H), (I, H), (H, I)))]
            g = x[b] @ m[0].T
            out[b] += 0.1 * s["w"].double()[b, k][:, None] * ((g * torch.sigmoid(g) * (x[b] @ m[1].T)) @ m[2].T)
        return out
    E, K = case["experts"], case["top_k"]
    rows = s["mask"].nonzero()[:, 0]
    z = s["logits"][rows].double()
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    ids = s["ids"][rows]
    counts = torch.bincount(ids[ids >= 0].long(), minlength=E)
    n = len(rows)
    f = counts.double() / (n * K)
    g = s["grad"].double()
    d = torch.zeros(case["tokens"], E, dtype=torch.float64, device="cuda")
    d[rows] = g[0] * E / n * p * (f - (p @ f)[:, None]) + g[1] * 2 / n * lse[:, None] * p
    return {"loss": torch.stack([E * (f * p.mean(0)).sum(), (lse ** 2).mean()]), "counts": counts.to(torch.int32), "dlogits": d}
