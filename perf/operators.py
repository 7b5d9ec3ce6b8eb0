"""The dense operators around a typed layer, over the sizes that users call them at.

A case is a dict of plain values; its "kind" names the operator:

  dropout   y = x / (1 - p) where a counter-based generator keeps the element,
            else 0; the mask is never stored (the backward pass is the same
            call on the gradient)
  norm      row LayerNorm with weights, followed by the same dropout: "fwd"
            gives the rows, "bwd" the gradients of the input, of the weight and
            of the bias, from the input rows and the seed alone
  grouped   products of rows sorted by group (the node types of a heterogeneous
            graph, the experts of a routed layer) with one matrix per group:
            "fwd" Y = X W_g, "bwd" both gradients dX = dY W_g^T and
            dW_g = X^T dY over the group's rows

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
        # The hidden rows of a small sampled subgraph: launch and latency count.
        dict(name="dropout_3k_f64", kind="dropout", n=3000, f=64, pad=0, dtype="f32", p=0.5),
        # Logit-wide rows of a citation-sized graph: 47 columns, rows that
        # start anywhere.
        dict(name="dropout_170k_f47", kind="dropout", n=170003, f=47, pad=0, dtype="f32", p=0.3),
        # The hidden rows of the product-shaped graph, in bf16.
        dict(name="dropout_product_bf16", kind="dropout", n=2449029, f=256, pad=0, dtype="bf16",
             p=0.5),
        # A handful of rows of a serving loop.
        dict(name="norm_serve_16x1024_bf16", kind="norm", pass_="fwd", n=16, f=1024, pad=0,
             dtype="bf16", p=0.0),
        # The hidden layer of the evaluation's model on the product-shaped
        # graph: 256 wide, dropout 0.5.
        dict(name="norm_product_fwd", kind="norm", pass_="fwd", n=2449029, f=256, pad=0,
             dtype="f32", p=0.5),
        # The backward pass at the input width of a citation-sized graph.
        dict(name="norm_170k_f100_bwd", kind="norm", pass_="bwd", n=170003, f=100, pad=0,
             dtype="f32", p=0.5),
        # The backward pass of the wide rows of a language model's batch.
        dict(name="norm_wide_bwd_bf16", kind="norm", pass_="bwd", n=16384, f=4096, pad=0,
             dtype="bf16", p=0.1),
        # Four node types of very different counts, each with its own projection
        # of the input features to the hidden width.
        dict(name="grouped_types_fwd", kind="grouped", pass_="fwd", n=500000, groups=4, empty=0,
             k=100, m=256, dtype="f32"),
        # The gradients of the hidden layer of the same graph.
        dict(name="grouped_types_bwd", kind="grouped", pass_="bwd", n=500000, groups=4, empty=0,
             k=256, m=256, dtype="f32"),
        # A large batch through sixteen wide expert matrices.
        dict(name="grouped_wide_fwd_bf16", kind="grouped", pass_="fwd", n=32768, groups=16,
             empty=0, k=2048, m=4096, dtype="bf16"),
        # Training with many small experts, some of which got no row.
        dict(name="grouped_many_bwd_bf16", kind="grouped", pass_="bwd", n=16384, groups=64,
             empty=5, k=1024, m=512, dtype="bf16"),
        # A few tokens of a serving loop spread over sixteen experts: the
        # matrices are read for one or two rows each.
        dict(name="grouped_serve_bf16", kind="grouped", pass_="fwd", n=24, groups=16, empty=3,
             k=2048, m=1024, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, hi):
    """A width: one of the configurations', a multiple of 8, or any."""
    return rng.choice([rng.choice([w for w in (47, 64, 100, 128, 256, 512, 1024, 4096) if w <= hi]),
                       8 * _log(rng, 4, hi // 8), _log(rng, 17, hi)])


def draw(rng):
    kind = rng.choice(["dropout", "norm", "norm", "grouped", "grouped", "grouped"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "dropout":
        f = _width(rng, 4096)
        return dict(kind=kind, n=_log(rng, 16, min(2449029, 300000000 // f)), f=f,
                    pad=rng.choice([0, 0, 8, rng.randint(1, 31)]), dtype=dtype,
                    p=rng.choice([0.1, 0.3, 0.5, rng.uniform(0.01, 0.9)]))
    if kind == "norm":
        f = _width(rng, 8192)
        return dict(kind=kind, pass_=rng.choice(["fwd", "bwd"]),
                    n=_log(rng, 4, min(2449029, 200000000 // f)), f=f,
                    pad=rng.choice([0, 0, 8, rng.randint(1, 31)]), dtype=dtype,
                    p=rng.choice([0.0, 0.1, 0.5, rng.uniform(0.01, 0.9)]))
    groups = _log(rng, 1, 128)
    k, m = _width(rng, 4096), _width(rng, 4096)
    while groups * k * m > 150000000:
        groups = max(1, groups // 2)
        k = max(k // 2, 17)
    most = min(500000, (15000000000 if dtype == "f32" else 120000000000) // (k * m))
    return dict(kind=kind, pass_=rng.choice(["fwd", "fwd", "bwd"]), n=_log(rng, 1, most),
                groups=groups, empty=rng.randint(0, groups // 4), k=k, m=m, dtype=dtype)


# ---- inputs --------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _rows(n, f, pad, dtype, g):
    """n rows of f normal values, pad columns apart."""
    x = torch.randn(n, f + pad, generator=g, device=DEV, dtype=torch.float32).to(dtype)
    return x[:, :f]


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


def prepare(case, seed):
    g = _gen(seed)
    dtype = TYPES[case["dtype"]]
    state = dict(case)
    if case["kind"] == "grouped":
        n, groups, k, m = (case[v] for v in ("n", "groups", "k", "m"))
        sizes = _sizes(n, groups, case["empty"], seed)
        ends = torch.cumsum(torch.tensor([0] + sizes), 0)
        state.update(sizes=sizes, offsets=ends.to(DEV),
                     w=(torch.randn(groups, k, m, generator=g, device=DEV)
                        / math.sqrt(k)).to(dtype))
        state["x"] = _rows(n, k, 0, dtype, g)
        if case["pass_"] == "bwd":
            state["dy"] = _rows(n, m, 0, dtype, g)
        return state
    state["x"] = _rows(case["n"], case["f"], case["pad"], dtype, g)
    state["seed"] = 0x1234567800000000 + seed
    state["call"] = seed % 5
    if case["kind"] == "norm":
        state["gamma"] = 1 + 0.2 * torch.randn(case["f"], generator=g, device=DEV)
        state["beta"] = 0.1 * torch.randn(case["f"], generator=g, device=DEV)
        state["eps"] = 1e-5
        if case["pass_"] == "bwd":
            state["dy"] = _rows(case["n"], case["f"], case["pad"], dtype, g)
    return state


# ---- the plain forms -----------------------------------------------------------

# Philox4x32 with 7 rounds (Salmon, Moraes, Dror, Shaw, "Parallel random
# numbers: as easy as 1, 2, 3", 2011): row i, columns 4 j .. 4 j + 3 take the four
# words of counter (j, i, call mod 2^32, call / 2^32) under the seed as key.
_LOW = 0xFFFFFFFF
_ROUNDS = 7


def _words(n, f, seed, call):
    """The 32-bit words of an n x f matrix, as int64."""
    c0 = torch.arange((f + 3) // 4, device=DEV)[None, :]
    c1 = torch.arange(n, device=DEV)[:, None]
    c2 = torch.full((1, 1), call & _LOW, device=DEV)
    c3 = torch.full((1, 1), call >> 32, device=DEV)
    k0, k1 = seed & _LOW, seed >> 32
    for _ in range(_ROUNDS):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # their 64 bits, as products modulo 2^64
        c0, c1, c2, c3 = (((b >> 32) & _LOW) ^ c1 ^ k0, b & _LOW,
                          ((a >> 32) & _LOW) ^ c3 ^ k1, a & _LOW)
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    return torch.stack([c.expand(n, (f + 3) // 4) for c in (c0, c1, c2, c3)], 2).view(n, -1)[:, :f]


def _drop(x, s):
    """x / (1 - p) where the element's word is at least p 2^32, else 0."""
    if s["p"] == 0.0:
        return x
    keep = _words(x.shape[0], x.shape[1], s["seed"], s["call"]) >= int(s["p"] * 4294967296.0)
    return torch.where(keep, x * (1.0 / (1.0 - s["p"])), torch.zeros((), device=DEV))


def _normalized(x, eps):
    d = x - x.mean(1, keepdim=True)
    rstd = torch.rsqrt(d.square().mean(1, keepdim=True) + eps)
    return d * rstd, rstd


def _plain(s):
    x = s["x"].float()
    t = s["x"].dtype
    if s["kind"] == "dropout":
        return _drop(x, s).to(t)
    if s["kind"] == "norm":
        h, rstd = _normalized(x, s["eps"])
        if s["pass_"] == "fwd":
            return _drop(h * s["gamma"] + s["beta"], s).to(t)
        g = _drop(s["dy"].float(), s)
        gg = g * s["gamma"]
        dx = rstd * (gg - gg.mean(1, keepdim=True) - h * (gg * h).mean(1, keepdim=True))
        return {"dx": dx.to(t), "dgamma": (g * h).sum(0), "dbeta": g.sum(0)}
    # one product per group, on the rows that it has
    w = s["w"].float()
    xs = torch.split(x, s["sizes"])
    if s["pass_"] == "fwd":
        return torch.cat([a @ b for a, b in zip(xs, w)]).to(t)
    gs = torch.split(s["dy"].float(), s["sizes"])
    return {"dx": torch.cat([a @ b.t() for a, b in zip(gs, w)]).to(t),
            "dw": torch.stack([a.t() @ b for a, b in zip(xs, gs)])}


def _library(s):
    import paper_2411_16025_amd as gcn
    if s["kind"] == "grouped":
        if s["pass_"] == "fwd":
            return gcn.gcn_gemm_grouped(gcn.GCN_GEMM_NN, s["offsets"], s["x"], s["w"])
        return {"dx": gcn.gcn_gemm_grouped(gcn.GCN_GEMM_NT, s["offsets"], s["dy"], s["w"]),
                "dw": gcn.gcn_gemm_grouped(gcn.GCN_GEMM_TN, s["offsets"], s["x"], s["dy"],
                                           out_dtype=torch.float32)}
    drop = gcn.Dropout(s["p"], s["seed"], s["call"]) if s["p"] else None
    if s["kind"] == "dropout":
        return gcn.gcn_dropout(s["x"], drop)
    if s["pass_"] == "fwd":
        return gcn.gcn_layernorm_affine_fwd(s["x"], s["gamma"], s["beta"], s["eps"], drop)
    dx, dgamma, dbeta = gcn.gcn_layernorm_affine_bwd(s["x"], s["dy"], s["gamma"], s["eps"], drop)
    return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta}


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    """Each input read once and each output written once; the products' operations
    (2 per multiplication), a few per element of the others."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "grouped":
        n, k, m, w = case["n"], case["k"], case["m"], case["groups"] - case["empty"]
        w = min(w, n) * k * m
        if case["pass_"] == "fwd":
            return {"bytes": e * (n * k + n * m + w), "flops": 2 * n * k * m}
        return {"bytes": e * (2 * n * k + n * m + w) + 4 * case["groups"] * k * m,
                "flops": 4 * n * k * m}
    n, f = case["n"], case["f"]
    if case["kind"] == "dropout":
        return {"bytes": 2 * e * n * f, "flops": n * f}
    if case["pass_"] == "fwd":
        return {"bytes": 2 * e * n * f + 8 * f, "flops": 8 * n * f}
    return {"bytes": 3 * e * n * f + 12 * f, "flops": 16 * n * f}


# ---- the definitions in 64 bits --------------------------------------------------


def _mul_words(a, m):
    """(high, low) 32-bit words of a * m by 16-bit halves of a."""
    lo, hi = (a % 65536) * m, (a // 65536) * m  # below 2^48
    mid = hi + lo // 65536
    return mid // 65536, (mid % 65536) * 65536 + lo % 65536


def _kept(rows, f, seed, call, p):
    """Which elements of the given rows are kept: word by word of the generator's
    definition, the four words of a counter in a state of four columns."""
    cols = (f + 3) // 4
    s = torch.empty(rows.numel(), cols, 4, dtype=torch.int64, device=DEV)
    s[:, :, 0] = torch.arange(cols, device=DEV)
    s[:, :, 1] = rows[:, None]
    s[:, :, 2] = call % 2**32
    s[:, :, 3] = call // 2**32
    for r in range(_ROUNDS):
        h0, l0 = _mul_words(s[:, :, 0], 3528531795)
        h2, l2 = _mul_words(s[:, :, 2], 3449720151)
        key0 = (seed % 2**32 + r * 2654435769) % 2**32
        key1 = (seed // 2**32 + r * 3144134277) % 2**32
        s = torch.stack([h2 ^ s[:, :, 1] ^ key0, l2, h0 ^ s[:, :, 3] ^ key1, l0], 2)
    return ~(s.reshape(rows.numel(), -1)[:, :f] < math.floor(p * 2.0**32))


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "grouped":
        ends = s["offsets"].tolist()
        y = torch.zeros(case["n"], case["m"] if case["pass_"] == "fwd" else case["k"],
                        dtype=torch.float64, device=DEV)
        dw = torch.zeros(case["groups"], case["k"], case["m"], dtype=torch.float64, device=DEV)
        for i in range(case["groups"]):
            rows = slice(ends[i], ends[i + 1])
            w = s["w"][i].double()
            if case["pass_"] == "fwd":
                y[rows] = s["x"][rows].double() @ w
            else:
                g = s["dy"][rows].double()
                y[rows] = g @ w.t().contiguous()
                dw[i] = s["x"][rows].double().t().contiguous() @ g
        return y if case["pass_"] == "fwd" else {"dx": y, "dw": dw}
    n, f, p = case["n"], case["f"], case["p"]
    out = torch.empty(n, f, dtype=torch.float64, device=DEV)
    dgamma = torch.zeros(f, dtype=torch.float64, device=DEV)
    dbeta = torch.zeros(f, dtype=torch.float64, device=DEV)
    step = max(1, 50000000 // f)
    for at in range(0, n, step):
        rows = torch.arange(at, min(n, at + step), device=DEV)
        x = s["x"][at:at + step].double()
        weight = torch.ones_like(x)
        if p:
            weight = _kept(rows, f, s["seed"], s["call"], p).double() / (1 - p)
        if case["kind"] == "dropout":
            out[at:at + step] = x * weight
            continue
        mean = x.sum(1, keepdim=True) / f
        std = torch.sqrt(((x - mean) ** 2).sum(1, keepdim=True) / f + s["eps"])
        h = (x - mean) / std
        if case["pass_"] == "fwd":
            out[at:at + step] = (h * s["gamma"].double() + s["beta"].double()) * weight
            continue
        g = s["dy"][at:at + step].double() * weight
        dgamma += (g * h).sum(0)
        dbeta += g.sum(0)
        g = g * s["gamma"].double()
        inner = g - g.sum(1, keepdim=True) / f - h * ((g * h).sum(1, keepdim=True) / f)
        out[at:at + step] = inner / std
    if case["kind"] == "norm" and case["pass_"] == "bwd":
        return {"dx": out, "dgamma": dgamma, "dbeta": dbeta}
    return out
