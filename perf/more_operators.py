"""Cases of the operators around the experts' products: inputs, plain forms in elementary torch
operations, the library's calls, and the definitions in 64 bits.

Four kinds of case (`op`):
  select    experts of every token from the router's logits: scores, bias, groups, top-K, weights; with
            `train` the gradient of the logits too
  dispatch  rows grouped by expert and copied into that order
  combine   the experts' rows back in the tokens' order, weighted, onto the residual; with `train` the gradients
  lora      low-rank adapters of many requests beside a shared projection; with `train` the gradients
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one token of a router with groups, on its way through a decode step: latency
        dict(name="select_token", op="select", tokens=1, experts=256, top_k=8, scores="sigmoid", bias=True, groups=8, top_groups=4,
             group_best=2, renorm=True, dtype="f32", train=False),
        # a training micro-batch of a plain softmax router, some rows padding
        dict(name="select_batch", op="select", tokens=4099, experts=64, top_k=6, scores="softmax", bias=False, groups=1, top_groups=1,
             group_best=1, renorm=False, dtype="f32", train=True),
        # the routing of a whole training batch
        dict(name="select_long", op="select", tokens=131072, experts=256, top_k=8, scores="sigmoid", bias=True, groups=8, top_groups=4,
             group_best=2, renorm=True, dtype="bf16", train=True),
        # a full decode batch on its way to small experts
        dict(name="dispatch_step", op="dispatch", tokens=64, experts=64, top_k=6, cols=2048, dtype="bf16"),
        # a long prefill over fine-grained experts
        dict(name="dispatch_long", op="dispatch", tokens=16384, experts=128, top_k=8, cols=2048, dtype="bf16"),
        # row lengths that no vector load fits
        dict(name="dispatch_odd", op="dispatch", tokens=3001, experts=5, top_k=3, cols=1413, dtype="f16"),
        # the end of a decode step: bf16 experts' rows onto an fp32 hidden state
        dict(name="combine_step", op="combine", tokens=64, experts=64, top_k=6, cols=2048, dtype="bf16", residual=True, train=False),
        # a training batch through large experts
        dict(name="combine_long", op="combine", tokens=16384, experts=8, top_k=2, cols=4096, dtype="bf16", residual=False, train=True),
        # fp16 rows of a width that is a multiple of nothing
        dict(name="combine_odd", op="combine", tokens=2047, experts=60, top_k=4, cols=1001, dtype="f16", residual=False, train=True),
        # a decode batch in which nearly every sequence brings an adapter of its own
        dict(name="lora_step", op="lora", tokens=64, adapters=64, rank=16, inner=4096, outer=4096, dtype="bf16", train=False),
        # prompts of a few requests beside the projection into a large expert
        dict(name="lora_prompts", op="lora", tokens=8192, adapters=5, rank=64, inner=4096, outer=14336, dtype="bf16", train=False),
        # adapters of three tenants trained together, at sizes of small experts
        dict(name="lora_train", op="lora", tokens=4099, adapters=3, rank=24, inner=2048, outer=2816, dtype="f16", train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["select", "dispatch", "combine", "lora"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if op == "select":
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * max(2, _log(rng, 2, 256) // groups)
        if experts > 256:
            experts = 256
        tokens = _log(rng, 1, 131072)
        top_groups = rng.randint(1, groups)
        top_k = min(top_groups * (experts // groups), _log(rng, 1, 16))
        scores = rng.choice(["softmax", "sigmoid"])
        bias = rng.random() < 0.5
        return dict(op=op, tokens=tokens, experts=experts, top_k=top_k, scores=scores, bias=bias, groups=groups, top_groups=top_groups,
                    group_best=2 if bias else 1, renorm=rng.random() < 0.5, dtype=dtype, train=rng.random() < 0.6)
    experts, top_k = _log(rng, 1, 256), _log(rng, 1, 8)
    if op == "lora":
        rank, inner, outer = _log(rng, 1, 128), _log(rng, 64, 8192), _log(rng, 64, 8192)
        tokens, adapters = _log(rng, 1, 8192), _log(rng, 1, 64)
        while tokens * (inner + 2 * outer) > 200_000_000:
            tokens //= 2
        return dict(op=op, tokens=tokens, adapters=adapters, rank=rank, inner=inner, outer=outer, dtype=rng.choice(["bf16", "f16"]),
                    train=rng.random() < 0.4)
    cols = _log(rng, 16, 8192)
    tokens = _log(rng, 1, max(2, min(32768, 100_000_000 // (cols * top_k))))
    case = dict(op=op, tokens=tokens, experts=max(experts, top_k), top_k=top_k, cols=cols, dtype=dtype)
    return case if op == "dispatch" else dict(case, residual=rng.random() < 0.5, train=rng.random() < 0.5)


# ---- inputs ----------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 2654435761 % (1 << 62))


def _activations(g, rows, cols, dtype):
    """Normal values with a few loud channels, as hidden states have them."""
    x = torch.randn(rows, cols, generator=g, device="cuda")
    loud = torch.rand(cols, generator=g, device="cuda") < 0.01
    return torch.where(loud, x * 20, x).to(dtype)


def _routing(g, T, E, K):
    """Ascending choices of top-K routing with uneven popularity; a few rows padding, a few choices dropped."""
    z = torch.randn(T, E, generator=g, device="cuda") + torch.randn(E, generator=g, device="cuda")
    ids = z.topk(K, 1).indices.sort(1).values.to(torch.int32)
    lost = torch.rand(T, K, generator=g, device="cuda") < 0.01
    lost |= (torch.rand(T, generator=g, device="cuda") < 0.05)[:, None]
    lost[0] = False
    return torch.where(lost, torch.full_like(ids, -1), ids).contiguous()


def prepare(case, seed):
    g = _gen(seed)
    op, dtype = case["op"], DTYPES[case["dtype"]]
    s = dict(case)
    T = case["tokens"]
    if op == "select":
        E, K = case["experts"], case["top_k"]
        z = (2 * torch.randn(T, E, generator=g, device="cuda") + torch.randn(E, generator=g, device="cuda")).to(dtype)
        s["mask"] = None
        if T > 8:
            z[3] = -math.inf                              # nothing left to choose
            z[5, 1:] = -math.inf                          # less than top_k left
            z[6, E // 2:] = torch.finfo(dtype).min        # a mask's fill value
            s["mask"] = torch.rand(T, generator=g, device="cuda") < 0.95
            s["mask"][3:7] = True
            z[~s["mask"]] = math.nan                      # padding holds anything
        s["logits"] = z
        s["offsets"] = 0.1 * torch.randn(E, generator=g, device="cuda") if case["bias"] else None
        s["grad"] = torch.randn(T, K, generator=g, device="cuda")
    elif op in ("dispatch", "combine"):
        K, C = case["top_k"], case["cols"]
        s["ids"] = _routing(g, T, case["experts"], K)
        if op == "dispatch":
            s["x"] = _activations(g, T, C, dtype)
            s["out"] = torch.zeros(T * K, C, dtype=dtype, device="cuda")   # kept; rows behind the last group stay 0
        else:
            s["plan"] = _plan(s["ids"], case["experts"])                   # made by the dispatch before
            s["y"] = _activations(g, T * K, C, dtype)
            s["w"] = torch.softmax(torch.randn(T, K, generator=g, device="cuda"), 1)
            s["h"] = torch.randn(T, C, generator=g, device="cuda") if case["residual"] else None
            s["grad"] = torch.randn(T, C, generator=g, device="cuda").to(torch.float32 if case["residual"] else dtype)
    else:
        n, r, I, O = (case[k] for k in ("adapters", "rank", "inner", "outer"))
        if T <= n:                                        # one token each, in any order
            ids = torch.randperm(n, generator=g, device="cuda")[:T].to(torch.int32)
            ids = torch.where(torch.rand(T, generator=g, device="cuda") < 0.1, torch.full_like(ids, -1), ids)
        else:                                             # prompts, one after the other, of uneven lengths
            cut = torch.rand(n, generator=g, device="cuda").sort().values * T
            ids = torch.searchsorted(cut, torch.arange(T, device="cuda").float()).to(torch.int32) - 1
        s["ids"] = ids
        s["plan"] = _plan(ids, n)                         # one for all projections of a step
        if not own:                                       # the plain form's plan: the rows of every adapter that has some
            s["rows"] = [(e, (ids == e).nonzero()[:, 0]) for e in sorted(set(ids.tolist())) if e >= 0]
        s["x"], s["base"] = _activations(g, T, I, dtype), _activations(g, T, O, dtype)
        s["a"] = (torch.randn(n, r, I, generator=g, device="cuda") / math.sqrt(I)).to(dtype)
        s["b"] = (0.05 * torch.randn(n, O, r, generator=g, device="cuda")).to(dtype)
        s["scale"] = 0.5 + torch.rand(n, generator=g, device="cuda")
        if case["train"]:
            s["grad"] = (0.1 * torch.randn(T, O, generator=g, device="cuda")).to(dtype)
    return s


def _plan(ids, n):
    """Which rows belong to which group: the library's plan, or its plain form."""
    if own:
        import paper_2606_15453_b200 as P
        return P.group_rows(ids, n)
    return _plain_group(ids, n)


# ---- one pass --------------------------------------------------------------------------------

def run(s):
    op = s["op"]
    if not own:
        return {"select": _plain_select, "dispatch": _plain_dispatch, "combine": _plain_combine, "lora": _plain_lora}[op](s)
    import paper_2606_15453_b200 as P
    if op == "select":
        f = P.router_select(s["logits"], s["top_k"], scores=s["scores"], bias=s["offsets"], groups=s["groups"], top_groups=s["top_groups"],
                            group_best=s["group_best"], renorm=s["renorm"], scale=2.5, mask=s["mask"])
        out = {"ids": f["ids"], "w": f["w"]}
        if s["train"]:
            out["dlogits"] = P.router_select_backward(s["logits"], f, s["grad"])
        return out
    if op == "dispatch":
        plan = P.group_rows(s["ids"], s["experts"])
        return {"counts": plan["counts"], "order": plan["order"], "slots": plan["slots"], "rows": P.dispatch_rows(s["x"], plan, out=s["out"])}
    if op == "combine":
        out = {"out": P.combine_rows(s["y"], s["plan"], s["w"], residual=s["h"], scale=0.1)}
        if s["train"]:
            out["dy"], out["dw"] = P.combine_rows_backward(s["grad"], s["y"], s["plan"], s["w"], scale=0.1)
        return out
    if not s["train"]:
        return {"out": P.lora(s["x"], s["a"], s["b"], s["plan"], scale=s["scale"], base=s["base"])}
    inner = torch.empty(s["tokens"], s["rank"], device="cuda")
    y = P.lora(s["x"], s["a"], s["b"], s["plan"], scale=s["scale"], base=s["base"], hidden=inner)
    dx, da, db = P.lora_backward(s["grad"], s["x"], s["a"], s["b"], s["plan"], inner, scale=s["scale"])
    return {"out": y, "dx": dx, "da": da, "db": db}


def _plain_keys(z, s):
    """Eligible choices' keys in 64 bits (values next to a border), -infinity where there is no choice."""
    z = z.double()
    if s["scores"] == "softmax":
        top = z.amax(1, keepdim=True)
        e = torch.exp(z - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
        score = e / e.sum(1, keepdim=True)
        if s["offsets"] is None and s["group_best"] == 1:
            score = z                                # the same order, also where scores underflow
    else:
        score = 1 / (1 + torch.exp(-z))
        if s["offsets"] is None and s["group_best"] == 1:
            score = z
    if s["offsets"] is not None:
        score = score + s["offsets"].double()
    return torch.where(z == -math.inf, torch.full_like(z, -math.inf), score)


def _plain_select(s):
    T, E, K, G = s["tokens"], s["experts"], s["top_k"], s["groups"]
    z = s["logits"].float()
    if s["mask"] is not None:
        z = torch.where(s["mask"][:, None], z, torch.full_like(z, -math.inf))
    key = _plain_keys(z, s)
    if G > 1:
        best = key.view(T, G, E // G).sort(2, descending=True).values[:, :, :min(s["group_best"], E // G)]
        best = best.sum(2)
        pick = best.sort(dim=1, descending=True, stable=True).indices[:, :s["top_groups"]]
        keep = torch.zeros(T, G, dtype=torch.bool, device=z.device).scatter_(1, pick, True)
        key = torch.where(keep.repeat_interleave(E // G, 1), key, torch.full_like(key, -math.inf))
    val, ids = key.sort(dim=1, descending=True, stable=True)
    ids = torch.where(val[:, :K] > -math.inf, ids[:, :K], torch.full_like(ids[:, :K], E)).sort(1).values
    there = ids < E
    at = torch.where(there, ids, torch.zeros_like(ids))
    zk = torch.where(there, z.gather(1, at), torch.full_like(z[:, :K], -math.inf))
    top = z.amax(1, keepdim=True)
    ex = torch.exp(z - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    tot = ex.sum(1, keepdim=True)
    tot = torch.where(tot > 0, tot, torch.ones_like(tot))
    soft = s["scores"] == "softmax"
    score = (ex.gather(1, at) / tot if soft else 1 / (1 + torch.exp(-zk))) * there
    if s["renorm"]:
        lk = zk if soft else torch.where(there, torch.clamp(zk, max=0) - torch.log1p(torch.exp(-zk.abs())), zk)
        lk = lk - torch.where(there[:, :1], lk.amax(1, keepdim=True), torch.zeros_like(lk[:, :1]))
        ek = torch.exp(lk) * there
        share = ek / ek.sum(1, keepdim=True).clamp(min=1)
    else:
        share = score
    out = {"ids": torch.where(there, ids, torch.full_like(ids, -1)).to(torch.int32), "w": 2.5 * share}
    if s["train"]:
        g = torch.where(there, 2.5 * s["grad"], torch.zeros_like(s["grad"]))
        slope = torch.where(there, 1 / (1 + torch.exp(zk)), torch.zeros_like(zk))           # 1 - sigmoid
        d = torch.zeros_like(z)
        if s["renorm"]:
            dk = share * (g - (share * g).sum(1, keepdim=True))
            dk = dk if soft else dk * slope
        else:
            dk = share * g if soft else share * slope * g
            if soft:
                d = -(ex / tot) * (share * g).sum(1, keepdim=True)
        d = torch.cat([d, d[:, :1]], 1).scatter_add(1, torch.where(there, ids, torch.full_like(ids, E)), dk)[:, :E]
        out["dlogits"] = d.to(s["logits"].dtype)
    return out


def _plain_group(ids, n):
    flat = ids.reshape(-1).long()
    flat = torch.where((flat >= 0) & (flat < n), flat, torch.full_like(flat, n))
    order = flat.sort(stable=True).indices
    slots = torch.empty_like(order)
    slots[order] = torch.arange(order.numel(), device=order.device)
    counts = torch.zeros(n + 1, dtype=torch.int64, device=ids.device).scatter_add(0, flat, torch.ones_like(flat))[:n]
    slots = torch.where(flat < n, slots, torch.full_like(slots, -1))
    return {"counts": counts.to(torch.int32), "order": order.to(torch.int32), "slots": slots.to(torch.int32).view(ids.shape)}


def _plain_dispatch(s):
    p = _plain_group(s["ids"], s["experts"])
    rows = s["x"].index_select(0, p["order"] // s["top_k"])
    there = torch.arange(rows.shape[0], device=rows.device) < p["counts"].sum()
    p["rows"] = torch.where(there[:, None], rows, s["out"])
    return p


def _plain_combine(s):
    slots, w, y = s["plan"]["slots"].long(), s["w"], s["y"]
    there = slots >= 0
    at = torch.where(there, slots, torch.zeros_like(slots))
    share = torch.where(there, 0.1 * w, torch.zeros_like(w))
    out = torch.zeros(s["tokens"], s["cols"], device=y.device) if s["h"] is None else s["h"].clone()
    for k in range(s["top_k"]):
        out += torch.where(there[:, k:k + 1], y[at[:, k]].float() * share[:, k:k + 1], torch.zeros_like(out))
    out = {"out": out.to(s["grad"].dtype)}
    if s["train"]:
        g = s["grad"].float()
        dy, dw = torch.zeros(y.shape[0] + 1, y.shape[1], device=y.device), torch.zeros_like(w)
        for k in range(s["top_k"]):
            dw[:, k] = torch.where(there[:, k], 0.1 * (g * y[at[:, k]].float()).sum(1), torch.zeros_like(dw[:, k]))
            rows = torch.where(there[:, k], slots[:, k], torch.full_like(slots[:, k], y.shape[0]))   # the last one: nobody's
            dy[rows] = torch.where(there[:, k:k + 1], g * share[:, k:k + 1], torch.zeros_like(g))
        out["dy"], out["dw"] = dy[:-1].to(y.dtype), dw
    return out


def _plain_lora(s):
    out = s["base"].float()
    x, a, b = s["x"].float(), s["a"].float(), s["b"].float()
    if s["train"]:
        g, dx, da, db = s["grad"].float(), torch.zeros_like(x), torch.zeros_like(a), torch.zeros_like(b)
    for e, rows in s["rows"]:
        xe = x[rows]
        he = torch.matmul(xe, a[e].t())
        out[rows] += s["scale"][e] * torch.matmul(he, b[e].t())
        if s["train"]:
            ge = s["scale"][e] * g[rows]
            te = torch.matmul(ge, b[e])
            dx[rows] = torch.matmul(te, a[e])
            da[e], db[e] = torch.matmul(te.t(), xe), torch.matmul(ge.t(), he)
    dt = s["x"].dtype
    if not s["train"]:
        return {"out": out.to(dt)}
    return {"out": out.to(dt), "dx": dx.to(dt), "da": da.to(dt), "db": db.to(dt)}


# ---- what a pass cannot do without ------------------------------------------------------------

def work(case):
    op, T, b = case["op"], case["tokens"], SIZE[case["dtype"]]
    if op == "select":
        E, K = case["experts"], case["top_k"]
        size = T * E * b + T * K * 8 + (E * 4 if case["bias"] else 0) + (T if T > 8 else 0)
        return {"bytes": size + (T * K * 4 + T * E * b if case["train"] else 0), "flops": T * E * (8 if case["train"] else 4)}
    if op == "lora":
        n, r, I, O = (case[k] for k in ("adapters", "rank", "inner", "outer"))
        used = min(n, T)
        size = b * (T * (I + 2 * O) + used * r * (I + O)) + T * 4
        flops = 2 * T * r * (I + O)
        if case["train"]:
            size += b * (T * (O + I) + n * r * (I + O))
            flops *= 3
        return {"bytes": size, "flops": flops}
    K, C = case["top_k"], case["cols"]
    if op == "dispatch":
        return {"bytes": T * C * b + T * K * C * b + 3 * T * K * 4 + case["experts"] * 4, "flops": T * K}
    o = 4 if case["residual"] else b
    size = T * K * C * b + T * K * 8 + T * C * o * (2 if case["residual"] else 1)
    if case["train"]:
        size += T * C * o + T * K * C * b + T * K * 4
    return {"bytes": size, "flops": T * K * C * (5 if case["train"] else 2)}


# ---- the definitions in 64 bits ----------------------------------------------------------------

def _exact_choice(key, K, G, top_groups, best):
    """One row at a time over all rows: K rounds of 'largest, lowest index first' on a copy of the keys."""
    T, E = key.shape
    key = key.clone()
    lowest = -math.inf
    if G > 1:
        left = key.view(T, G, E // G).clone()
        total = torch.zeros(T, G, dtype=torch.float64, device=key.device)
        for _ in range(min(best, E // G)):
            top, at = left.max(2)
            total += top
            left.scatter_(2, at[:, :, None], lowest)
        allowed = torch.zeros(T, G, dtype=torch.bool, device=key.device)
        for _ in range(top_groups):
            # the first of the largest, also among groups that have nothing
            open_ = ~allowed
            top = torch.where(open_, total, torch.full_like(total, lowest)).amax(1, keepdim=True)
            first = ((total == top) & open_).to(torch.int32).argmax(1)
            allowed[torch.arange(T, device=key.device), first] = True
        key = torch.where(allowed.repeat_interleave(E // G, 1), key, torch.full_like(key, lowest))
    chosen = torch.zeros(T, E, dtype=torch.bool, device=key.device)
    for _ in range(K):
        top = key.amax(1, keepdim=True)
        hit = (key == top) & (top > lowest)
        first = hit.to(torch.int32).argmax(1, keepdim=True)
        hit = torch.zeros_like(hit).scatter_(1, first, hit.gather(1, first))
        chosen |= hit
        key[hit] = lowest
    return chosen


def _exact_select(s):
    T, E, K = s["tokens"], s["experts"], s["top_k"]
    z = s["logits"].double()
    if s["mask"] is not None:
        z[~s["mask"]] = -math.inf
    soft = s["scores"] == "softmax"
    live = (z > -math.inf).any(1)
    logp = torch.zeros_like(z)
    logp[live] = torch.log_softmax(z[live], 1) if soft else -torch.logaddexp(torch.zeros_like(z[live]), -z[live])
    logp[~(z > -math.inf)] = -math.inf
    if s["offsets"] is None and s["group_best"] == 1:
        key = z
    else:
        key = torch.exp(logp) + (0 if s["offsets"] is None else s["offsets"].double())
        key = torch.where(z > -math.inf, key, torch.full_like(key, -math.inf))
    chosen = _exact_choice(key, K, s["groups"], s["top_groups"], s["group_best"])
    # columns of the chosen in ascending order, E where none is left
    cols = torch.where(chosen, torch.arange(E, device=z.device).expand(T, E), torch.full((T, E), E, device=z.device)).sort(1).values[:, :K]
    there = cols < E
    wide = torch.where(chosen, logp, torch.full_like(logp, -math.inf))
    if s["renorm"]:
        some = chosen.any(1)
        share = torch.zeros_like(wide)
        share[some] = torch.softmax(wide[some], 1)
    else:
        share = torch.exp(wide)
    pad = torch.cat([share, torch.zeros_like(share[:, :1])], 1)
    out = {"ids": torch.where(there, cols, torch.full_like(cols, -1)).to(torch.int32), "w": 2.5 * pad.gather(1, cols)}
    if s["train"]:
        g = torch.zeros(T, E + 1, dtype=torch.float64, device=z.device).scatter_(1, cols, 2.5 * s["grad"].double())[:, :E]
        g = torch.where(chosen, g, torch.zeros_like(g))
        mean = (share * g).sum(1, keepdim=True)
        if soft:
            d = share * (g - mean) if s["renorm"] else share * g - torch.exp(logp) * mean
        else:
            d = share * (g - mean if s["renorm"] else g) * torch.where(chosen, torch.sigmoid(-z), torch.zeros_like(z))
        out["dlogits"] = d
    return out


def _exact_plan(ids, n):
    """Counting, group by group."""
    flat = ids.reshape(-1)
    order, slots = [], torch.full_like(flat, -1)
    counts, at = [], 0
    for e in range(n):
        rows = (flat == e).nonzero()[:, 0].to(torch.int32)
        slots[rows.long()] = torch.arange(at, at + rows.numel(), dtype=torch.int32, device=ids.device)
        at += rows.numel()
        order.append(rows)
        counts.append(rows.numel())
    order.append(((flat < 0) | (flat >= n)).nonzero()[:, 0].to(torch.int32))
    return {"counts": torch.tensor(counts, dtype=torch.int32, device=ids.device), "order": torch.cat(order), "slots": slots.view(ids.shape)}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "select":
        return _exact_select(s)
    if op == "dispatch":
        p = _exact_plan(s["ids"], case["experts"])
        n = int(p["counts"].sum())
        p["rows"] = s["out"].clone()
        p["rows"][:n] = s["x"][p["order"][:n].long() // case["top_k"]]
        return p
    if op == "combine":
        T, K, C = case["tokens"], case["top_k"], case["cols"]
        slots = _exact_plan(s["ids"], case["experts"])["slots"].long()
        t, k = (slots >= 0).nonzero(as_tuple=True)
        rows = slots[t, k]
        out = torch.zeros(T, C, dtype=torch.float64, device="cuda") if s["h"] is None else s["h"].double()
        dy = torch.zeros(T * K, C, dtype=torch.float64, device="cuda") if case["train"] else None
        dw = torch.zeros(T, K, dtype=torch.float64, device="cuda")
        for j in range(K):
            m = k == j
            out[t[m]] += 0.1 * s["w"].double()[t[m], j][:, None] * s["y"].double()[rows[m]]
            if case["train"]:
                g = s["grad"].double()[t[m]]
                dy[rows[m]] = 0.1 * s["w"].double()[t[m], j][:, None] * g
                dw[t[m], j] = 0.1 * (g * s["y"].double()[rows[m]]).sum(1)
        return {"out": out, "dy": dy, "dw": dw} if case["train"] else {"out": out}
    out = s["base"].double()
    if case["train"]:
        dx, da, db = (torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (s["x"], s["a"], s["b"]))
    for e in range(case["adapters"]):
        at = (s["ids"] == e).nonzero()[:, 0]
        if at.numel() == 0:
            continue
        x, a, b = s["x"][at].double(), s["a"][e].double(), s["b"][e].double()
        c = float(s["scale"][e])
        out[at] += c * ((x @ a.T) @ b.T)
        if case["train"]:
            g = c * s["grad"][at].double()
            dx[at] = (g @ b) @ a
            da[e], db[e] = (g @ b).T @ x, g.T @ (x @ a.T)
    return {"out": out, "dx": dx, "da": da, "db": db} if case["train"] else {"out": out}
