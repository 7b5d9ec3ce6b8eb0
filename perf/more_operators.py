"""The operators that bring rows to a typed or routed layer and back, over their sizes.

A case is a dict of plain values; its "kind" names the operator:

  embed      rows of a learned table: "fwd" Y[i] = scale * T[ids[i]] (ids of -1
             give zeros), "bwd" the table's gradient, summed by sorted ids
  route      the k largest logits of each row, their softmax weights, the rows
             per expert and the balance loss
             E * coef * sum_e (c_e / sum c) (mean_t p_te); "bwd" the logits'
             gradient from that of the weights and of the loss
  dispatch   positions sorted by expert and the rows in that order: what the
             products by group read
  combine    Y[t] = sum_i w[t, i] Z[slot[t, i]]; "bwd" the gradients of Z and w
  keep8      rows kept in 8 bits (codes of 32 columns under one power of two)
             and brought back
  grad8      products by group dW_g = X_g^T dY_g from the rows kept so

`run` computes them in elementary operations, or, where `own` is true, by the
library's calls. Every input is drawn on the GPU from the seed.
"""

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # The rows of a few ids of a serving loop: launch and latency count.
        dict(name="embed_serve_24", kind="embed", pass_="fwd", n=24, table=50000, f=1024, skew=1,
             pad=0, dtype="bf16", out="bf16"),
        # Learned inputs of the product-shaped graph's nodes: a sampled batch's
        # gradient, most rows of the table without any.
        dict(name="embed_nodes_bwd", kind="embed", pass_="bwd", n=250000, table=2449029, f=100,
             skew=1, pad=0, dtype="f32", out="f32"),
        # A batch of tokens, of which a few ids are a large part.
        dict(name="embed_tokens_bwd_bf16", kind="embed", pass_="bwd", n=131072, table=50000,
             f=1024, skew=4, pad=4096, dtype="bf16", out="f32"),
        # One small batch through a router of sixteen experts.
        dict(name="route_serve_64", kind="route", pass_="fwd", n=64, experts=16, k=2, closed=0,
             pad=0, normalize=True, dtype="f32"),
        # A large batch with many small experts, the last rows padding.
        dict(name="route_128k_fwd_bf16", kind="route", pass_="fwd", n=131072, experts=64, k=8,
             closed=0, pad=1000, normalize=True, dtype="bf16"),
        # The gradient over more experts than a wavefront has lanes.
        dict(name="route_32k_bwd", kind="route", pass_="bwd", n=32768, experts=256, k=4, closed=5,
             pad=0, normalize=False, dtype="f32"),
        # The rows of that router's batch in the experts' order.
        dict(name="dispatch_32k_bf16", kind="dispatch", n=32768, experts=16, k=2, f=2048,
             dtype="bf16"),
        # Back to the tokens' order, eight small experts each.
        dict(name="combine_16k_k8_bf16", kind="combine", pass_="fwd", n=16384, k=8, f=1024, drop=0,
             dtype="bf16"),
        # The gradients, some choices dropped.
        dict(name="combine_32k_bwd_bf16", kind="combine", pass_="bwd", n=32768, k=2, f=2048,
             drop=700, dtype="bf16"),
        # The hidden rows of the product-shaped graph, kept for the backward pass.
        dict(name="keep8_product", kind="keep8", n=2449029, f=256, pad=0, dtype="f32"),
        # The weight gradients of four node types' input projections.
        dict(name="grad8_types", kind="grad8", n=500000, groups=4, empty=0, k=100, m=256,
             dtype="f32"),
        # Those of sixteen wide experts.
        dict(name="grad8_wide_bf16", kind="grad8", n=32768, groups=16, empty=1, k=2048, m=4096,
             dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, hi):
    """A width: one of the configurations', a multiple of 8, or any."""
    return rng.choice([rng.choice([w for w in (47, 64, 100, 128, 256, 512, 1024, 4096) if w <= hi]),
                       8 * _log(rng, 4, hi // 8), _log(rng, 17, hi)])


def draw(rng):
    kind = rng.choice(["embed", "embed", "route", "route", "dispatch", "combine", "combine",
                       "keep8", "grad8", "grad8"])
    dtype = rng.choice(["f32", "bf16"])
    pass_ = rng.choice(["fwd", "bwd"])
    if kind == "embed":
        f = _width(rng, 4096)
        n = _log(rng, 1, min(1000000, 130000000 // f))
        table = _log(rng, 2, min(2449029, 240000000 // f))
        return dict(kind=kind, pass_=pass_, n=n, table=table, f=f, skew=rng.choice([1, 1, 2, 4]),
                    pad=rng.choice([0, 0, rng.randint(0, n // 4)]), dtype=dtype,
                    out=rng.choice(["f32", "bf16"]))
    if kind == "route":
        experts = rng.choice([8, 16, 64, 128, 256, _log(rng, 2, 512)])
        n = _log(rng, 1, min(200000, 16000000 // experts))
        return dict(kind=kind, pass_=pass_, n=n, experts=experts,
                    k=rng.randint(1, min(8, experts)),
                    closed=rng.choice([0, 0, rng.randint(0, experts // 4)]),
                    pad=rng.choice([0, 0, rng.randint(0, n // 4)]),
                    normalize=rng.random() < 0.5, dtype=dtype)
    if kind == "dispatch":
        f, k = _width(rng, 4096), rng.randint(1, 8)
        return dict(kind=kind, n=_log(rng, 1, min(200000, 120000000 // (f * k))),
                    experts=_log(rng, 1, 512), k=k, f=f, dtype=dtype)
    if kind == "combine":
        f, k = _width(rng, 4096), rng.randint(1, 8)
        n = _log(rng, 1, min(200000, 100000000 // (f * k)))
        return dict(kind=kind, pass_=pass_, n=n, k=k, f=f,
                    drop=rng.choice([0, rng.randint(0, n * k // 4)]), dtype=dtype)
    if kind == "keep8":
        f = _width(rng, 4096)
        return dict(kind=kind, n=_log(rng, 4, min(2449029, 600000000 // f)), f=f,
                    pad=rng.choice([0, 0, 8, rng.randint(1, 31)]), dtype=dtype)
    groups = _log(rng, 1, 128)
    k, m = _width(rng, 4096), _width(rng, 4096)
    while groups * k * m > 150000000:
        groups = max(1, groups // 2)
        k = max(k // 2, 17)
    most = min(500000, (20000000000 if dtype == "f32" else 120000000000) // (k * m))
    return dict(kind=kind, n=_log(rng, 1, most), groups=groups, empty=rng.randint(0, groups // 4),
                k=k, m=m, dtype=dtype)


# ---- inputs --------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rows(n, f, pad, dtype, g):
    """n rows of f normal values, pad columns apart."""
    x = torch.randn(n, f + pad, generator=g, device=DEV, dtype=torch.float32).to(dtype)
    return x[:, :f]


def _uniform(n, g):
    return torch.rand(n, generator=g, device=DEV, dtype=torch.float64)


def _sizes(n, groups, empty, seed):
    """How the n rows fall to the groups: shares of very different size,
    `empty` groups without any."""
    g = torch.Generator()
    g.manual_seed(seed)
    share = torch.rand(groups, generator=g, dtype=torch.float64) ** 2 + 0.02
    share[torch.randperm(groups, generator=g)[:empty]] = 0.0
    ends = torch.round(torch.cumsum(share, 0) / share.sum() * n).to(torch.int64)
    ends[-1] = n
    return torch.diff(ends, prepend=torch.zeros(1, dtype=torch.int64)).tolist()


def _choices(n, experts, k, g):
    """k different experts for each of n rows, the first ones taken more often."""
    lean = torch.linspace(1.0, 0.0, experts, device=DEV)
    score = torch.randn(n, experts, generator=g, device=DEV) + lean
    return torch.argsort(score, 1, descending=True)[:, :k].to(torch.int32)


def prepare(case, seed):
    g = _gen(seed)
    kind, n = case["kind"], case["n"]
    dtype = TYPES[case["dtype"]]
    state = dict(case)
    if kind == "embed":
        ids = (_uniform(n, g) ** case["skew"] * case["table"]).to(torch.int32)
        ids = ids.clamp_(max=case["table"] - 1)
        if case["pad"]:
            ids[torch.randperm(n, generator=g, device=DEV)[:case["pad"]]] = -1
        state.update(ids=ids, scale=math.sqrt(case["f"]))
        if case["pass_"] == "fwd":
            state["t"] = _rows(case["table"], case["f"], 0, dtype, g)
        else:
            state["dy"] = _rows(n, case["f"], 0, dtype, g)
        return state
    if kind == "route":
        z = 1.5 * torch.randn(n, case["experts"], generator=g, device=DEV)
        z[:, torch.randperm(case["experts"], generator=g, device=DEV)[:case["closed"]]] = -math.inf
        z = z.to(dtype)
        mask = None
        if case["pad"]:
            mask = torch.ones(n, dtype=torch.uint8, device=DEV)
            mask[n - case["pad"]:] = 0
        state.update(z=z, mask=mask, coef=0.01)
        if case["pass_"] == "bwd":  # what the forward pass gave
            state.update(zip(("chosen", "weights", "counts"), _plain_route(state)[:3]))
            state["dw"] = torch.randn(n, case["k"], generator=g, device=DEV) / n
        return state
    if kind == "dispatch":
        state["experts_of"] = _choices(n, case["experts"], case["k"], g)
        state["x"] = _rows(n, case["f"], 0, dtype, g)
        return state
    if kind == "combine":
        m = n * case["k"]
        # the places of the choices sorted by expert, the dropped ones behind them all
        ids = _choices(n, 64, case["k"], g).flatten()
        ids[torch.randperm(m, generator=g, device=DEV)[:case["drop"]]] = 64
        order = torch.argsort(ids, stable=True)
        slot = torch.empty(m, dtype=torch.int32, device=DEV)
        slot[order] = torch.arange(m, dtype=torch.int32, device=DEV)
        slot[ids == 64] = -1
        w = torch.rand(n, case["k"], generator=g, device=DEV) + 0.05
        state.update(slot=slot.view(n, case["k"]), w=w / w.sum(1, keepdim=True),
                     z=_rows(m, case["f"], 0, dtype, g))
        if case["pass_"] == "bwd":
            state["dy"] = _rows(n, case["f"], 0, dtype, g)
            # (the dropped choices' rows keep what they hold)
            state["dz"] = torch.zeros(m, case["f"], dtype=dtype, device=DEV)
        return state
    if kind == "keep8":
        state["x"] = _rows(n, case["f"], case["pad"], dtype, g)
        return state
    sizes = _sizes(n, case["groups"], case["empty"], seed)
    ends = torch.cumsum(torch.tensor([0] + sizes), 0)
    codes, scales = _pack(_rows(n, case["k"], 0, dtype, g).float())
    state.update(sizes=sizes, offsets=ends.to(DEV), codes=codes, scales=scales,
                 dy=_rows(n, case["m"], 0, dtype, g))
    return state


# ---- the plain forms -----------------------------------------------------------


def _plain_embed(s):
    out = TYPES[s["out"]]
    ids = s["ids"].long()
    real = ids >= 0
    if s["pass_"] == "fwd":
        y = s["t"][ids.clamp(min=0)].float() * s["scale"]
        return torch.where(real[:, None], y, torch.zeros((), device=DEV)).to(out)
    dt = torch.zeros(s["table"], s["f"], device=DEV)
    dt.index_add_(0, ids[real], s["dy"][real].float())
    return (dt * s["scale"]).to(out)


def _softmax(z):
    """Rows of -inf alone give zeros."""
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - torch.where(top == -math.inf, torch.zeros_like(top), top))
    return e / e.sum(1, keepdim=True).clamp(min=1e-30)


def _plain_route(s):
    """(experts, weights, counts and how many rows count, loss)"""
    z = s["z"].float()
    experts = s["experts"]
    if s["mask"] is not None:
        z = torch.where(s["mask"][:, None] > 0, z, torch.full((), -math.inf, device=DEV))
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :s["k"]]
    p = _softmax(z)
    open_ = z.gather(1, order) > -math.inf
    w = torch.where(open_, p.gather(1, order), torch.zeros((), device=DEV))
    if s["normalize"]:
        w = w / w.sum(1, keepdim=True).clamp(min=1e-30)
    chosen = torch.where(open_, order, torch.full_like(order, -1))
    counts = (chosen[:, :, None] == torch.arange(experts, device=DEV)).sum((0, 1)) \
        if chosen.numel() * experts < 1 << 24 else \
        torch.stack([(chosen == e).sum() for e in range(experts)])
    rows = open_[:, 0].sum()
    share = counts.double() / counts.sum().clamp(min=1)
    mean = p.double().sum(0) / rows.clamp(min=1)
    loss = (s["coef"] * experts * (share * mean).sum()).float()
    return chosen.to(torch.int32), w, torch.cat([counts, rows[None]]), loss


def _plain_route_bwd(s):
    z = s["z"].float()
    experts = s["experts"]
    counts, rows = s["counts"][:-1], s["counts"][-1]
    open_ = s["chosen"] >= 0
    p = torch.where(open_[:, :1], _softmax(z), torch.zeros((), device=DEV))
    at = s["chosen"].long().clamp(min=0)
    g = torch.where(open_, s["dw"], torch.zeros((), device=DEV))
    a = s["coef"] * experts * counts.float() / (counts.sum() * rows).clamp(min=1).float()
    dz = p * (a - (p * a).sum(1, keepdim=True))
    w = s["weights"]
    inner = (g * w).sum(1, keepdim=True)
    if s["normalize"]:
        dz = dz.scatter_add(1, at, w * (g - inner))
    else:
        dz = (dz - p * inner).scatter_add(1, at, w * g)
    return dz.to(s["z"].dtype)


def _plain_dispatch(s):
    ids = s["experts_of"].flatten().long()
    order = torch.argsort(ids, stable=True)
    slot = torch.empty_like(order)
    slot[order] = torch.arange(ids.numel(), device=DEV)
    ends = (ids[order][:, None] <= torch.arange(s["experts"], device=DEV)).sum(0) \
        if ids.numel() * s["experts"] < 1 << 26 else \
        torch.stack([(ids <= e).sum() for e in range(s["experts"])])
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), ends])
    return {"offsets": offsets, "order": order.to(torch.int32), "slot": slot.to(torch.int32),
            "x": s["x"][order // s["k"]]}


def _plain_combine(s):
    t = s["z"].dtype
    slot = s["slot"].long()
    real = slot >= 0
    w = torch.where(real, s["w"], torch.zeros((), device=DEV))
    if s["pass_"] == "fwd":
        y = torch.zeros(s["n"], s["f"], device=DEV)
        for i in range(s["k"]):
            y += w[:, i:i + 1] * s["z"][slot[:, i].clamp(min=0)].float()
        return y.to(t)
    dy = s["dy"].float()
    dw = torch.empty_like(s["w"])
    dz = s["dz"]
    for i in range(s["k"]):
        at = slot[:, i]
        dw[:, i] = torch.where(real[:, i], (dy * s["z"][at.clamp(min=0)].float()).sum(1),
                               torch.zeros((), device=DEV))
        rows = real[:, i].nonzero()[:, 0]
        dz[at[rows]] = (w[rows, i:i + 1] * dy[rows]).to(t)
    return {"dz": dz, "dw": dw}


def _pack(x):
    """Codes and scale bytes of fp32 rows: blocks of 32 columns hold q 2^(b - 127), b the
    smallest in [1, 248] that keeps |q| at 127 or less."""
    n, f = x.shape
    blocks = (f + 31) // 32
    if blocks * 32 != f:
        x = torch.cat([x, torch.zeros(n, blocks * 32 - f, device=DEV)], 1)
    x = x.view(n, blocks, 32)
    top = x.abs().amax(2)
    m, e = torch.frexp(top)  # top = m 2^e, m in [0.5, 1)
    e = torch.where(top > 0, e - 7 + (m > 127 / 128).int(), torch.full_like(e, -126))
    e = e.clamp(-126, 121)
    q = torch.round(torch.ldexp(x, -e[:, :, None])).clamp(-127, 127)
    return (q.view(n, -1)[:, :f].to(torch.int8).contiguous(),
            (e + 127).to(torch.uint8).contiguous())


def _unpack(codes, scales):
    e = scales.int().repeat_interleave(32, 1)[:, :codes.shape[1]] - 127
    return torch.ldexp(codes.float(), e)


def _plain(s):
    kind = s["kind"]
    if kind == "embed":
        return _plain_embed(s)
    if kind == "route":
        if s["pass_"] == "bwd":
            return _plain_route_bwd(s)
        return dict(zip(("experts", "weights", "counts", "loss"), _plain_route(s)))
    if kind == "dispatch":
        return _plain_dispatch(s)
    if kind == "combine":
        return _plain_combine(s)
    if kind == "keep8":
        return _unpack(*_pack(s["x"].float())).to(s["x"].dtype)
    xs = torch.split(_unpack(s["codes"], s["scales"]), s["sizes"])
    return torch.stack([a.t() @ b for a, b in zip(xs, torch.split(s["dy"].float(), s["sizes"]))])


def _library(s):
    import paper_2411_16025_amd as gcn
    kind = s["kind"]
    if kind == "embed":
        out = TYPES[s["out"]]
        if s["pass_"] == "fwd":
            return gcn.gcn_embed_fwd(s["t"], s["ids"], scale=s["scale"], out_dtype=out)
        offsets, order, _ = gcn.gcn_group_ids(s["ids"], s["table"], slots=False)
        return gcn.gcn_embed_bwd(s["dy"], offsets, order, scale=s["scale"], out_dtype=out)
    if kind == "route":
        if s["pass_"] == "bwd":
            return gcn.gcn_route_bwd(s["z"], s["chosen"], s["weights"], s["counts"], dweights=s["dw"],
                                     coef=s["coef"], normalize=s["normalize"])
        chosen, weights, counts, loss = gcn.gcn_route_fwd(s["z"], s["k"], mask=s["mask"],
                                                          coef=s["coef"], normalize=s["normalize"])
        return {"experts": chosen, "weights": weights, "counts": counts, "loss": loss}
    if kind == "dispatch":
        offsets, order, slot = gcn.gcn_group_ids(s["experts_of"].view(-1), s["experts"])
        return {"offsets": offsets, "order": order, "slot": slot,
                "x": gcn.gcn_embed_fwd(s["x"], order, per=s["k"])}
    if kind == "combine":
        if s["pass_"] == "fwd":
            return gcn.gcn_combine_fwd(s["z"], s["slot"], s["w"])
        dz, dw = gcn.gcn_combine_bwd(s["z"], s["slot"], s["w"], s["dy"], dZ=s["dz"])
        return {"dz": dz, "dw": dw}
    if kind == "keep8":
        codes, scales = gcn.gcn_pack8(s["x"])
        return gcn.gcn_unpack8(codes, scales, out_dtype=s["x"].dtype)
    return gcn.gcn_gemm_grouped_q8(s["offsets"], s["codes"], s["scales"], s["dy"])


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    """Each input read once and each output written once; the products' operations
    (2 per multiplication), a few per element of the others."""
    kind, n = case["kind"], case["n"]
    e = 4 if case["dtype"] == "f32" else 2
    if kind == "embed":
        f, out = case["f"], 4 if case["out"] == "f32" else 2
        if case["pass_"] == "fwd":
            return {"bytes": 4 * n + min(n, case["table"]) * f * e + n * f * out, "flops": n * f}
        return {"bytes": 4 * n + (n - case["pad"]) * f * e + case["table"] * f * out,
                "flops": n * f}
    if kind == "route":
        rows = n * case["experts"] * e * (2 if case["pass_"] == "bwd" else 1)
        return {"bytes": rows + n * case["k"] * (12 if case["pass_"] == "bwd" else 8),
                "flops": 8 * n * case["experts"]}
    if kind == "dispatch":
        m = n * case["k"]
        return {"bytes": 12 * m + (n + m) * case["f"] * e, "flops": m}
    if kind == "combine":
        m = n * case["k"] - case["drop"]
        if case["pass_"] == "fwd":
            return {"bytes": 8 * m + (m + n) * case["f"] * e, "flops": 2 * m * case["f"]}
        return {"bytes": 12 * m + (2 * m + n) * case["f"] * e, "flops": 3 * m * case["f"]}
    if kind == "keep8":
        return {"bytes": 2 * n * case["f"] * e, "flops": 4 * n * case["f"]}
    k, m = case["k"], case["m"]
    return {"bytes": n * k + n * ((k + 31) // 32) + n * m * e + 4 * case["groups"] * k * m,
            "flops": 2 * n * k * m}


# ---- the definitions in 64 bits --------------------------------------------------


def _exact_embed(case, s):
    f, ids = case["f"], s["ids"].long()
    if case["pass_"] == "fwd":
        y = torch.zeros(case["n"], f, dtype=torch.float64, device=DEV)
        rows = torch.nonzero(ids != -1)[:, 0]
        y[rows] = s["t"].double()[ids[rows]] * s["scale"]
        return y
    # the running sum of the sorted rows, a few columns at a time, taken at each id's end
    order = torch.argsort(ids)
    keys = ids[order].contiguous()
    ends = torch.searchsorted(keys, torch.arange(-1, case["table"], device=DEV), right=True)
    dt = torch.empty(case["table"], f, dtype=torch.float64, device=DEV)
    zero = torch.zeros(1, 1, dtype=torch.float64, device=DEV)
    step = max(1, 100000000 // max(case["n"], case["table"]))
    for at in range(0, f, step):
        g = s["dy"][:, at:at + step].double()[order]
        sums = torch.cat([zero.expand(1, g.shape[1]), torch.cumsum(g, 0)])
        dt[:, at:at + step] = (sums[ends[1:]] - sums[ends[:-1]]) * s["scale"]
    return dt


def _exact_route(case, s):
    z = s["z"].double()
    n, experts, k = case["n"], case["experts"], case["k"]
    masked = torch.isinf(z)
    if s["mask"] is not None:
        masked = masked | (s["mask"] == 0)[:, None]
    e = torch.where(masked, torch.zeros_like(z), torch.exp(z))  # (the logits are small numbers)
    total = e.sum(1, keepdim=True)
    p = torch.where(total > 0, e / total, torch.zeros_like(e))
    if case["pass_"] == "bwd":
        chosen, counts = s["chosen"].long(), s["counts"].double()
        dp = torch.zeros(n, experts + 1, dtype=torch.float64, device=DEV)
        g = s["dw"].double()
        at = torch.where(chosen >= 0, chosen, torch.full_like(chosen, experts))
        if case["normalize"]:
            pc = torch.cat([p, torch.zeros(n, 1, dtype=torch.float64, device=DEV)], 1).gather(1, at)
            sel = pc.sum(1, keepdim=True)
            g = g / sel - (g * pc).sum(1, keepdim=True) / sel ** 2
        dp.scatter_(1, at, g)
        dp = dp[:, :experts] + s["coef"] * experts * counts[:-1] / (counts[:-1].sum() * counts[-1])
        dz = p * (dp - (p * dp).sum(1, keepdim=True))
        return torch.where(chosen[:, :1] >= 0, dz, torch.zeros_like(dz))
    left = torch.where(masked, torch.full_like(z, -math.inf), z)
    chosen, w = [], []
    index = torch.arange(experts, device=DEV)
    for _ in range(k):  # the lowest index among the largest
        top = left.amax(1, keepdim=True)
        i = torch.where(left == top, index, torch.full_like(index, experts)).amin(1)
        none = top[:, 0] == -math.inf
        w.append(torch.where(none, torch.zeros_like(top[:, 0]), p.gather(1, i[:, None])[:, 0]))
        chosen.append(torch.where(none, torch.full_like(i, -1), i))
        left = left.scatter(1, i[:, None], -math.inf)
    chosen, w = torch.stack(chosen, 1), torch.stack(w, 1)
    if case["normalize"]:
        w = torch.where(w > 0, w / w.sum(1, keepdim=True), torch.zeros_like(w))
    counts = torch.bincount(chosen.flatten() + 1, minlength=experts + 1)[1:]
    rows = (chosen[:, 0] >= 0).sum()
    loss = s["coef"] * experts * (counts.double() * p.sum(0)).sum() / (counts.sum() * rows)
    return {"experts": chosen.to(torch.int32), "weights": w,
            "counts": torch.cat([counts, rows[None]]), "loss": loss}


def exact(case, seed):
    s = prepare(case, seed)
    kind, n = case["kind"], case["n"]
    if kind == "embed":
        return _exact_embed(case, s)
    if kind == "route":
        return _exact_route(case, s)
    if kind == "dispatch":
        ids = s["experts_of"].flatten().long()
        keys, order = torch.sort(ids * ids.numel() + torch.arange(ids.numel(), device=DEV))
        offsets = torch.searchsorted(keys, torch.arange(case["experts"] + 1, device=DEV)
                                     * ids.numel())
        slot = torch.searchsorted(keys, ids * ids.numel() + torch.arange(ids.numel(), device=DEV))
        return {"offsets": offsets, "order": order.to(torch.int32), "slot": slot.to(torch.int32),
                "x": s["x"].double().repeat_interleave(case["k"], 0)[order]}
    if kind == "combine":
        slot = s["slot"].flatten().long()
        rows = torch.nonzero(slot != -1)[:, 0]
        w, token = s["w"].double().flatten(), rows // case["k"]
        z = torch.zeros(n * case["k"], case["f"], dtype=torch.float64, device=DEV)
        z[rows] = s["z"].double()[slot[rows]]
        if case["pass_"] == "fwd":
            return (z * w[:, None]).view(n, case["k"], -1).sum(1)
        dy = s["dy"].double()
        dz = torch.zeros_like(z)
        dz[slot[rows]] = w[rows, None] * dy[token]
        return {"dz": dz, "dw": (z.view(n, case["k"], -1) * dy[:, None, :]).sum(2)}
    if kind == "keep8":
        y = torch.empty(n, case["f"], dtype=torch.float64, device=DEV)
        step = max(1, 50000000 // case["f"])
        for at in range(0, n, step):
            for c in range(0, case["f"], 32):
                x = s["x"][at:at + step, c:c + 32].double()
                top = x.abs().amax(1, keepdim=True)
                unit = torch.exp2(torch.ceil(torch.log2(top / 127)).clamp(-126, 121))
                # (where the logarithm's rounding put the unit beside the smallest one)
                unit = torch.where(top > 127 * unit, unit * 2, unit)
                unit = torch.where((top <= 63.5 * unit) & (unit > 2.0 ** -126), unit / 2, unit)
                y[at:at + step, c:c + 32] = torch.round(x / unit).clamp(-127, 127) * unit
        return y
    ends = s["offsets"].tolist()
    dw = torch.zeros(case["groups"], case["k"], case["m"], dtype=torch.float64, device=DEV)
    block = torch.arange(case["k"], device=DEV) // 32
    for i in range(case["groups"]):
        rows = slice(ends[i], ends[i + 1])
        x = s["codes"][rows].double() * torch.exp2(s["scales"][rows].double() - 127)[:, block]
        dw[i] = x.t().contiguous() @ s["dy"][rows].double()
    return dw
