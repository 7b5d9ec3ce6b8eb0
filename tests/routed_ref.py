"""References of the routed layer's operators in 64 bits (host, numpy), and checks of the library's calls
against them. The checks take an engine: memory for arrays, and the library's entry points (the GPU's in
test_gpu_routed.py, the kernels on the CPU in test_routed_model.py)."""

import ctypes
import math

import numpy as np

from gpu_util import bf16_round

U = 2.0 ** -24         # half a step of fp32
HALF = {"f32": 0.0, "bf16": 2.0 ** -8}  # half a step of a type, relative (fp32's is counted with the sums)
CODE = {"f32": 0, "bf16": 1}


def rounded(x, kind):
    x = np.asarray(x, np.float32)
    return bf16_round(x) if kind == "bf16" else x


class Call:
    """The scratch memory modes of a call: the library's, or the caller's of just the size asked for."""

    def __init__(self, engine, memory):
        self.engine, self.memory = engine, memory

    def __call__(self, f, *args):
        e = self.engine
        if not self.memory:
            st = f(*args, None, None, e.stream)
        else:
            need = ctypes.c_int64(-1)
            assert f(*args, None, ctypes.byref(need), e.stream) == 0
            assert need.value >= 0 and need.value % 256 == 0
            some = need.value > 0  # (without memory and with its size, the call would ask again)
            st = f(*args, e.work(need.value) if some else None, ctypes.byref(need) if some else None, e.stream)
        assert st == 0, (f, st, e.error())


# ---- positions by group ------------------------------------------------------------


def group_ids(ids, G):
    ids = np.asarray(ids, np.int64)
    key = np.where((ids >= 0) & (ids < G), ids, G)
    order = np.argsort(key, kind="stable")
    offsets = np.searchsorted(key[order], np.arange(G + 1))
    slot = np.empty(len(ids), np.int64)
    slot[order] = np.arange(len(ids))
    return offsets, np.where(key[order] < G, order, -1), np.where(key < G, slot, -1)


def some_ids(r, n, G, how):
    """ids: spread, a few very often, all the same, or some that belong to no group."""
    if how == "one":
        return np.full(n, G // 2, np.int32)
    ids = (r.random(n) ** (4 if how == "skew" else 1) * G).astype(np.int64)
    if how == "none":
        out = r.random(n) < 0.3
        ids[out] = r.choice(np.array([-1, G, -2 ** 31, 2 ** 31 - 1]), out.sum())
    return ids.astype(np.int32)


def check_group_ids(e, n, G, how, memory=0, seed=0, only=None):
    r = np.random.default_rng(seed)
    ids = some_ids(r, n, G, how)
    i, o = e.put(ids), e.new((G + 1,), np.int64)
    order, slot = e.new((n,), np.int32), e.new((n,), np.int32)
    Call(e, memory)(e.lib.gcn_group_ids, n, i.ptr, G, o.ptr, None if only == "slot" else order.ptr,
                    None if only == "order" else slot.ptr)
    want = group_ids(ids, G)
    for got, w, nm in zip((o, order, slot), want, ("offsets", "order", "slot")):
        if only in (None, nm) or nm == "offsets":
            assert np.array_equal(got.get(), w), (nm, n, G, how)


# ---- rows of a table ---------------------------------------------------------------


def check_embed_fwd(e, n, F, V, per=1, kt="f32", ky="f32", pad=0, shift=0, scale=1.7, seed=0):
    r = np.random.default_rng(seed)
    T = rounded(r.standard_normal((V, F)), kt)
    ids = some_ids(r, n, V * per, "none")
    used = np.zeros(V, bool)
    used[ids[(ids >= 0) & (ids.astype(np.int64) < V * per)] // per] = True
    T[~used] = np.nan
    t, y = e.rows(T, kt, pad, shift), e.rows(np.full((n, F), 7.0), ky, pad + 1, shift, fill=9.0)
    i = e.put(ids)
    assert e.lib.gcn_embed_fwd(n, F, V, i.ptr, per, t.ptr, t.ld, CODE[kt], scale, y.ptr, y.ld, CODE[ky],
                               e.stream) == 0, e.error()
    real = (ids >= 0) & (ids.astype(np.int64) < V * per)
    at = np.where(real, ids, 0) // per
    want = rounded(np.where(real[:, None], np.float32(scale) * np.nan_to_num(T[at]), np.float32(0)), ky)
    got = y.get()
    assert np.array_equal(got, want), (n, F, V, per, kt, ky)
    assert not np.signbit(got[~real]).any()
    y.check_margins()


def check_embed_bwd(e, n, F, V, how="spread", kd="f32", kt="f32", pad=0, shift=0, add=False, memory=0,
                    scale=-0.6, seed=0):
    r = np.random.default_rng(seed)
    dY = rounded(r.standard_normal((n, F)), kd)
    ids = some_ids(r, n, V, how)
    offsets, order, slots = group_ids(ids, V)
    dY[slots < 0] = np.nan  # (of no row of the table)
    old = rounded(r.standard_normal((V, F)), kt)
    dy = e.rows(dY, kd, max(pad, 0), shift)
    dt = e.rows(old if add else np.full((V, F), np.nan), kt, pad + 2, shift, fill=9.0)
    o, p = e.put(offsets.astype(np.int64)), e.put(order.astype(np.int32))
    Call(e, memory)(e.lib.gcn_embed_bwd, n, F, V, o.ptr, p.ptr, dy.ptr, dy.ld, CODE[kd], scale, dt.ptr,
                    dt.ld, CODE[kt], 1 if add else 0)
    ref, mag, count = np.zeros((V, F)), np.zeros((V, F)), np.zeros(V)
    for j, v in zip(order[:offsets[V]], np.repeat(np.arange(V), np.diff(offsets))):
        ref[v] += dY[j].astype(np.float64)
        mag[v] += np.abs(dY[j])
        count[v] += 1
    s = float(np.float32(scale))
    # a chain of at most 256 additions (and the first chunk's, in the join), the sum and the scale rounded
    # once, the sum with what was there once, and half a step of the type
    bound = (np.minimum(count, 256)[:, None] + 4) * U * abs(s) * mag
    want = s * ref
    if add:
        want = want + np.where(count[:, None] > 0, old, old)
        bound = bound + U * np.abs(want)
        bound[count == 0] = 0
    got = dt.get().astype(np.float64)
    touched = (count > 0)[:, None]
    bound = bound + np.where(touched, HALF[kt] * (np.abs(want) + bound), 0)
    bad = ~(np.abs(got - want) <= bound)
    assert not bad.any(), (n, F, V, how, kd, kt, np.argwhere(bad)[:3], got[bad][:3], want[bad][:3])
    dt.check_margins()
    return dt


# ---- the router --------------------------------------------------------------------


def softmax(z):
    """p of the rows, zeros of rows of -inf alone."""
    z = np.asarray(z, np.float64)
    m = z.max(1, keepdims=True)
    with np.errstate(invalid="ignore"):
        x = np.where(np.isneginf(z), -np.inf, z - np.where(np.isneginf(m), 0, m))
    ex = np.exp(x)
    s = ex.sum(1, keepdims=True)
    return ex / np.where(s > 0, s, 1), x


def route(z, k, mask, normalize):
    """(experts, weights, counts, p, relative error bounds of p in units of U)"""
    z = np.array(z, np.float64)
    n, E = z.shape
    if mask is not None:
        z[mask == 0] = -np.inf
    p, x = softmax(z)
    order = np.argsort(-z, axis=1, kind="stable")[:, :k]
    none = np.isneginf(np.take_along_axis(z, order, 1))
    w = np.where(none, 0, np.take_along_axis(p, order, 1))
    if normalize:
        s = w.sum(1, keepdims=True)
        w = w / np.where(s > 0, s, 1)
    experts = np.where(none, -1, order)
    counts = np.zeros(E + 1, np.int64)
    np.add.at(counts, np.where(none, E, order).ravel(), 1)
    counts[E] = (~none[:, 0]).sum()
    # z - max is rounded once, which exp turns into as many U as it is large; exp and the products 4 U; the
    # sum over a row of chains of 16 and 6 joins, whose terms have those errors too
    far = np.where(np.isneginf(x), 0, -x)
    rel = far + (p * far).sum(1, keepdims=True) + 40
    return experts, w, counts, p, rel


def some_logits(r, n, E, kind, how):
    z = rounded(r.standard_normal((n, E)) * 2, kind)
    if how == "ties":  # few different values
        z = np.round(z).astype(np.float32)
    if how == "closed":
        z[r.random((n, E)) < 0.6] = -np.inf
    if how == "far":
        z = rounded(z * 30, kind)
    return z


def check_route(e, n, E, k, kind="f32", how="plain", normalize=False, masked=False, coef=0.02, pad=0,
                shift=0, memory=0, loss=True, seed=0):
    """Forward, then backward from the reference's outputs."""
    r = np.random.default_rng(seed)
    z = some_logits(r, n, E, kind, how)
    mask = (r.random(n) < 0.7).astype(np.uint8) if masked else None
    zd = e.rows(z, kind, pad, shift)
    md = e.put(mask) if masked else None
    ex, w = e.new((n, k), np.int32), e.new((n, k), np.float32)
    counts, ls = e.new((E + 1,), np.int64), e.new((1,), np.float32)
    Call(e, memory)(e.lib.gcn_route_fwd, n, E, zd.ptr, zd.ld, CODE[kind], k, 1 if normalize else 0,
                    md.ptr if masked else None, coef, ex.ptr, w.ptr, counts.ptr, ls.ptr if loss else None)
    experts, weights, cnt, p, rel = route(z, k, mask, normalize)
    what = (n, E, k, kind, how, normalize, masked)
    assert np.array_equal(ex.get(), experts), what
    assert np.array_equal(counts.get(), cnt), what
    # normalized: the quotient by the sum of at most 64 chosen ones, with their errors
    wrel = np.where(experts >= 0, np.take_along_axis(rel, np.maximum(experts, 0), 1), 0)
    wrel = 2 * wrel.max(1, keepdims=True) + 70 if normalize else wrel
    assert (np.abs(w.get() - weights) <= wrel * U * weights + 1e-37).all(), what
    if loss:
        c, N = cnt[:E].astype(np.float64), cnt[E]
        want = coef * E * (c * p.sum(0)).sum() / (c.sum() * N) if N else 0.0
        # the rows of a lane one after the other (512 workgroups of at least 4 rows share them), 6 joins
        depth = n / 2048 + 10
        bound = coef * E * (c * ((rel + depth) * p).sum(0)).sum() / max(c.sum() * N, 1) * U + U * abs(want)
        assert abs(float(ls.get()[0]) - want) <= bound + 1e-37, (what, ls.get(), want)
    # backward
    dw = r.standard_normal((n, k)).astype(np.float32)
    wf = weights.astype(np.float32)
    dl = np.float32(1.3)
    dz = e.rows(np.full((n, E), 7.0), kind, pad + 1, shift, fill=9.0)
    ed, wd, cd, gd, ld = (e.put(v) for v in (experts.astype(np.int32), wf, cnt, dw, np.array([dl])))
    assert e.lib.gcn_route_bwd(n, E, zd.ptr, zd.ld, CODE[kind], k, 1 if normalize else 0, ed.ptr, wd.ptr,
                               cd.ptr, coef, gd.ptr, ld.ptr, dz.ptr, dz.ld, e.stream) == 0, e.error()
    want, bound = route_grad(z, experts, wf, cnt, dw, coef, float(dl), normalize, p, rel)
    bound = bound + HALF[kind] * (np.abs(want) + bound)
    got = dz.get()
    bad = ~(np.abs(got - want) <= bound + 1e-37)
    assert not bad.any(), (what, np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], bound[bad][:3])
    dz.check_margins()


def route_grad(z, experts, w, counts, dw, coef, dloss, normalize, p=None, rel=None):
    n, E = z.shape
    k = experts.shape[1]
    if p is None:
        p, _ = softmax(z)
        rel = np.zeros_like(p)
    real = experts >= 0
    p = np.where(real[:, :1], p, 0)
    g, w = np.where(real, dw, 0).astype(np.float64), np.asarray(w, np.float64)
    a = coef * E * dloss * counts[:E] / max(counts[:E].sum() * counts[E], 1)
    inner = (g * w).sum(1, keepdims=True)
    size = (np.abs(g * w)).sum(1, keepdims=True)
    dz, mag = np.zeros((n, E)), np.zeros((n, E))
    rows, cols = np.nonzero(real)
    at = experts[rows, cols]
    x = w * (g - inner) if normalize else w * g
    np.add.at(dz, (rows, at), x[rows, cols])
    m = np.abs(w) * (np.abs(g) + size) if normalize else np.abs(w * g)
    np.add.at(mag, (rows, at), m[rows, cols])
    A = (p * a).sum(1, keepdims=True)
    rest = a - A - (0 if normalize else inner)
    dz += p * rest
    # p with its errors; the sums over the row and the choices 40 + k roundings of their magnitudes
    size = np.abs(a) + np.abs(A) + (0 if normalize else size)
    worst = rel.max(1, keepdims=True)
    bound = U * ((k + 40) * mag + p * ((rel + 8) * size + (worst + 40 + k) * size))
    return dz, bound


# ---- back from the groups' order ------------------------------------------------------


def some_slots(r, n, k, rows):
    """Different places for the choices, some choices dropped."""
    m = n * k
    slot = np.full(m, -1, np.int64)
    take = min(m, rows)
    slot[r.permutation(m)[:take]] = r.permutation(rows)[:take]
    drop = r.random(m) < 0.15
    slot[drop] = r.choice(np.array([-1, rows, -2 ** 31, 2 ** 31 - 1]), drop.sum())
    return slot.astype(np.int32).reshape(n, k)


def check_combine(e, n, k, F, rows, kind="f32", weighted=True, pad=0, shift=0, in_place=False, seed=0):
    """Forward and backward."""
    r = np.random.default_rng(seed)
    Z, dY = rounded(r.standard_normal((rows, F)), kind), rounded(r.standard_normal((n, F)), kind)
    slot = some_slots(r, n, k, rows)
    w = r.standard_normal((n, k)).astype(np.float32)
    real = (slot >= 0) & (slot < rows)
    at = np.where(real, slot, 0)
    used = np.zeros(rows, bool)
    used[slot[real]] = True
    Z[~used] = np.nan
    W = np.where(real, w if weighted else 1, 0).astype(np.float64)
    z, y = e.rows(Z, kind, pad, shift), e.rows(np.full((n, F), 7.0), kind, pad + 1, shift, fill=9.0)
    sd, wd = e.put(slot), e.put(w)
    what = (n, k, F, rows, kind, weighted)
    assert e.lib.gcn_combine_fwd(n, k, F, z.ptr, rows, z.ld, CODE[kind], sd.ptr, wd.ptr if weighted else None,
                                 y.ptr, y.ld, e.stream) == 0, e.error()
    Zk = np.where(real[:, :, None], Z[at], 0) if rows else np.zeros((n, k, F), np.float32)
    terms = W[:, :, None] * Zk
    want, bound = terms.sum(1), (k + 1) * U * np.abs(terms).sum(1)
    bound = bound + HALF[kind] * (np.abs(want) + bound)
    got = y.get()
    assert (np.abs(got - want) <= bound).all(), what
    assert not np.signbit(got[~real.any(1)]).any()
    y.check_margins()
    # backward
    dy = e.rows(dY, kind, pad, shift)
    dz = z if in_place else e.rows(np.full((rows, F), 5.0), kind, pad + 1, shift, fill=9.0)
    dw = e.new((n, k), np.float32)
    assert e.lib.gcn_combine_bwd(n, k, F, z.ptr, rows, z.ld, CODE[kind], sd.ptr, wd.ptr if weighted else None,
                                 dy.ptr, dy.ld, dz.ptr, dz.ld, dw.ptr, e.stream) == 0, e.error()
    want = Z.copy() if in_place else np.full((rows, F), 5.0, np.float32)
    t, i = np.nonzero(real)
    want[slot[t, i]] = rounded((w[t, i] if weighted else np.ones(len(t), np.float32))[:, None] * dY[t], kind)
    assert np.array_equal(dz.get(), want, equal_nan=True), what
    terms = np.where(real[:, :, None], Zk.astype(np.float64) * dY[:, None, :], 0)
    # at least 8 lanes share a row: chains of F / 8 + 8, six joins
    bound = (F / 8 + 24) * U * np.abs(terms).sum(2)
    assert (np.abs(dw.get() - terms.sum(2)) <= bound).all(), what
    dz.check_margins()


# ---- rows in 8 bits ----------------------------------------------------------------


def pack8(x):
    """(codes, scale bytes) by the definition."""
    x = np.asarray(x, np.float64)
    n, F = x.shape
    B = (F + 31) // 32
    q, s = np.zeros((n, F), np.int8), np.zeros((n, B), np.uint8)
    for b in range(B):
        v = x[:, 32 * b:32 * b + 32]
        bad = ~np.isfinite(v).all(1)
        top = np.where(bad, 0, np.abs(np.where(np.isfinite(v), v, 0)).max(1))
        e = np.full(n, 121)
        for c in range(120, -127, -1):
            e = np.where(top <= 127 * 2.0 ** c, c, e)
        with np.errstate(invalid="ignore"):
            code = np.clip(np.rint(v * (2.0 ** -e.astype(np.float64))[:, None]), -127, 127)
        q[:, 32 * b:32 * b + 32] = np.where(bad[:, None], 0, np.nan_to_num(code)).astype(np.int8)
        s[:, b] = np.where(bad, 255, e + 127)
    return q, s


def unpack8(q, s):
    unit = np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127))
    return q.astype(np.float64) * np.repeat(unit, 32, 1)[:, :q.shape[1]]


def some_rows(r, n, F, kind, how):
    x = r.standard_normal((n, F))
    if how == "sizes":  # of very different size, down to denormal numbers and up to the largest
        x = x * 2.0 ** r.integers(-149, 126, (n, (F + 31) // 32)).repeat(32, 1)[:, :F]
    if how == "edges":  # 127 2^c, what lies beside it, halves between codes, zeros
        x = r.choice(np.array([127.0, np.nextafter(np.float32(127), 0), np.nextafter(np.float32(127), 200),
                               127.5, 128.0, 63.5, 0.5, 1.5, 2.5, -2.5, 0.0, -0.0, -127.0]), (n, F))
        x = x * 2.0 ** r.integers(-20, 20, (n, 1))
    if how == "special":
        x = np.where(r.random((n, F)) < 0.02, r.choice(np.array([np.inf, -np.inf, np.nan, 3.4e38, 1e-45]),
                                                         (n, F)), x)
    with np.errstate(over="ignore"):
        return rounded(x.astype(np.float32), kind)


def check_pack8(e, n, F, kind="f32", how="plain", pad=0, shift=0, seed=0):
    r = np.random.default_rng(seed)
    x = some_rows(r, n, F, kind, how)
    B = (F + 31) // 32
    xd = e.rows(x, kind, pad, shift)
    q = e.rows(np.full((n, F), 99), "i8", pad + 1, shift, fill=77)
    s = e.rows(np.full((n, B), 99), "u8", pad, shift, fill=77)
    assert e.lib.gcn_pack8(n, F, xd.ptr, xd.ld, CODE[kind], q.ptr, q.ld, s.ptr, s.ld, e.stream) == 0, e.error()
    wq, ws = pack8(x)
    what = (n, F, kind, how, pad, shift)
    assert np.array_equal(s.get(), ws), what
    assert np.array_equal(q.get(), wq), what
    q.check_margins()
    s.check_margins()
    for ky in ("f32", "bf16"):
        y = e.rows(np.full((n, F), 7.0), ky, pad, shift, fill=9.0)
        assert e.lib.gcn_unpack8(n, F, q.ptr, q.ld, s.ptr, s.ld, y.ptr, y.ld, CODE[ky], e.stream) == 0
        want = unpack8(wq, ws)
        assert np.array_equal(y.get().astype(np.float64), want, equal_nan=True), what
        y.check_margins()


def check_grad8(e, sizes, K, N, kind="f32", before=0, after=0, pad=0, memory=0, whole=True, seed=0):
    """whole: small whole numbers, sums exact; else within the roundings of a chain of sums."""
    r = np.random.default_rng(seed)
    G = len(sizes)
    ends = before + np.concatenate([[0], np.cumsum(sizes)])
    rows = int(ends[-1] + after)
    B = (K + 31) // 32
    if whole:
        q = r.integers(-3, 4, (rows, K)).astype(np.int8)
        s = r.integers(126, 129, (rows, B)).astype(np.uint8)
        b = r.integers(-3, 4, (rows, N)).astype(np.float32)
    else:
        q, s = pack8(r.standard_normal((rows, K)))
        b = rounded(r.standard_normal((rows, N)), kind)
    member = np.zeros(rows, bool)
    member[ends[0]:ends[-1]] = True
    s[~member] = 255
    b[~member] = np.nan
    qd, sd = e.rows(q, "i8", pad, fill=77), e.rows(s, "u8", pad, fill=255)
    bd = e.rows(b, kind, pad)
    c = e.rows(np.full((G * K, N), 7.0), "f32", pad, fill=9.0)
    o = e.put(ends.astype(np.int64))
    Call(e, memory)(e.lib.gcn_gemm_grouped_q8, G, o.ptr, rows, N, K, qd.ptr, qd.ld, sd.ptr, sd.ld, bd.ptr, bd.ld,
                    CODE[kind], c.ptr, c.ld, K * c.ld)
    got = c.get().reshape(G, K, N)
    what = (sizes if G < 9 else (G, rows), K, N, kind, pad, memory)
    for g in range(G):
        rng = slice(ends[g], ends[g + 1])
        x, y = unpack8(q[rng], s[rng]), b[rng].astype(np.float64)
        want = x.T @ y
        if whole:
            assert np.array_equal(got[g], want), (what, g, np.argwhere(got[g] != want)[:4])
        else:
            # sums of at most 65536 products in chains, the partial ones in double; the products 4 U
            bound = (min(sizes[g], 65536) + 8) * U * (np.abs(x).T @ np.abs(y))
            assert (np.abs(got[g] - want) <= bound).all(), (what, g)
    c.check_margins()


def check_grad8_special(e, rows, K, N, kind="f32", seed=0):
    """Rows of B with infinities, NaN, the largest and the smallest numbers, and rows of X that stand for NaN:
    in whole columns, so that sums have one value whatever their order."""
    r = np.random.default_rng(seed)
    q, s = pack8(r.standard_normal((rows, K)))
    b = rounded(r.standard_normal((rows, N)), kind)
    one = np.zeros((rows, N), np.float32)
    one[rows // 2] = 1
    b[:, 0] = np.where(one[:, 0] > 0, np.inf, 0)  # sums are infinite, or NaN where q is 0
    b[rows // 3, 1] = np.nan
    b[:, 2] = one[:, 2] * rounded(3.3e38, kind)
    b[:, 3] *= np.float32(2.0 ** -120)     # (and their lower parts denormal numbers)
    b[:, 4] = rounded(b[:, 4] * np.float32(2.0 ** 100), kind)
    b[:, 5] = 0
    s[rows - 1, 0] = 255
    q[rows - 1, :32] = 0
    qd, sd, bd = e.rows(q, "i8", 0), e.rows(s, "u8", 0), e.rows(b, kind, 0)
    c, o = e.rows(np.full((K, N), 7.0), "f32", 0), e.put(np.array([0, rows], np.int64))
    Call(e, 0)(e.lib.gcn_gemm_grouped_q8, 1, o.ptr, rows, N, K, qd.ptr, qd.ld, sd.ptr, sd.ld, bd.ptr, bd.ld,
               CODE[kind], c.ptr, c.ld, K * N)
    got, x = c.get(), unpack8(q, s)
    with np.errstate(invalid="ignore", over="ignore"):
        want = x.T @ b.astype(np.float64)
        mag = np.abs(x).T @ np.abs(b.astype(np.float64))
    what = (rows, K, N, kind)
    assert np.isnan(got[:32]).all() and np.isnan(got[:, 1]).all(), what
    rest = slice(32, K)
    # bf16 multiplies denormal numbers' lower parts by nothing: its products are exact, but those below 2^-126
    # and their sums may be lost (8-bit values times 2^-120 normal ones are above 2^-133 times 127)
    tiny = rows * 2.0 ** -126 if kind == "bf16" else rows * 2.0 ** -149
    with np.errstate(invalid="ignore", over="ignore"):
        near = np.abs(got - want) <= (rows + 8) * U * mag + tiny
        big = np.abs(want) > 3.4e38
    assert np.array_equal(np.isnan(got[rest, 0]), x[rows // 2, rest] == 0), what
    assert np.array_equal(np.isinf(got[rest, 0]), x[rows // 2, rest] != 0), what
    ok = near | (big & np.isinf(got) & (np.sign(got) == np.sign(want)))
    assert ok[rest, 2:].all(), (what, np.argwhere(~ok[rest, 2:])[:4])
    assert (got[rest, 5] == 0).all() and not np.signbit(got[rest, 5]).any(), what


def check_embed_bwd_unordered(e, n, F, V, kd="f32", seed=0):
    """Offsets and an order of any values: nothing is read or written outside of the arrays."""
    r = np.random.default_rng(seed)
    dY = rounded(r.standard_normal((n, F)), kd)
    offsets = np.where(r.random(V + 1) < 0.8, r.integers(0, n + 1, V + 1), r.integers(-2 ** 62, 2 ** 62, V + 1))
    order = np.where(r.random(n) < 0.8, r.integers(0, n, n), r.integers(-2 ** 31, 2 ** 31, n))
    dy, dt = e.rows(dY, kd, 1), e.rows(np.zeros((V, F)), "f32", 1, fill=9.0)
    o, p = e.put(offsets.astype(np.int64)), e.put(order.astype(np.int32))
    for memory in (0, 1):
        Call(e, memory)(e.lib.gcn_embed_bwd, n, F, V, o.ptr, p.ptr, dy.ptr, dy.ld, CODE[kd], 1.0, dt.ptr, dt.ld, 0, 0)
    dt.check_margins()


def check_grad8_unordered(e, G, rows, K, N, kind="f32", seed=0):
    r = np.random.default_rng(seed)
    offsets = np.where(r.random(G + 1) < 0.8, r.integers(0, rows + 1, G + 1), r.integers(-2 ** 62, 2 ** 62, G + 1))
    q, s = pack8(r.standard_normal((rows, K)))
    qd, sd = e.rows(q, "i8", 0), e.rows(s, "u8", 0)
    bd, c = e.rows(rounded(r.standard_normal((rows, N)), kind), kind, 0), e.rows(np.zeros((G * K, N)), "f32", 0)
    o = e.put(offsets.astype(np.int64))
    for memory in (0, 1):
        Call(e, memory)(e.lib.gcn_gemm_grouped_q8, G, o.ptr, rows, N, K, qd.ptr, qd.ld, sd.ptr, sd.ld, bd.ptr, bd.ld,
                        CODE[kind], c.ptr, c.ld, K * c.ld)


def check_route_bwd_any(e, n, E, k, kind="f32", seed=0):
    """Experts of any values: nothing is read or written outside of the arrays."""
    r = np.random.default_rng(seed)
    z = e.rows(rounded(r.standard_normal((n, E)), kind), kind, 1)
    ex = e.put(r.integers(-2 ** 31, 2 ** 31, (n, k)).astype(np.int32) >> r.integers(0, 31, (n, k)).astype(np.int32))
    w, c = e.put(r.random((n, k)).astype(np.float32)), e.put(r.integers(0, 9, E + 1))
    dz = e.rows(np.zeros((n, E)), kind, 1, fill=9.0)
    assert e.lib.gcn_route_bwd(n, E, z.ptr, z.ld, CODE[kind], k, 1, ex.ptr, w.ptr, c.ptr, 1.0, w.ptr, None, dz.ptr,
                               dz.ld, e.stream) == 0
    dz.check_margins()


def check_grad8_scales(e, sizes, K, N, kind="f32", small=-10, large=None, seed=0):
    """Rows of X at both ends of the scale bytes: the first 32 columns with finite values up to the largest ones
    (bytes 247 and 248, codes of 0 and of all sizes under them), the last block of columns with the smallest (byte
    1). B is of size 2^small, from column N / 2 on 2^large where that is given."""
    r = np.random.default_rng(seed)
    rows = int(np.sum(sizes))
    x = r.standard_normal((rows, K))
    last = (K - 1) // 32 * 32
    top = r.choice(np.array([2e38, -2e38, 3.3e38, -3.3e38, 1e38, -1e38]), rows)
    at = r.integers(0, min(K, 32), rows)
    big = r.random(rows) < 0.4
    big[:2] = True, rows < 2
    x[big, at[big]] = top[big]
    spread = big & (r.random(rows) < 0.5)  # codes of all sizes beside it
    c = slice(0, min(K, 32))
    x[spread, c] = r.uniform(-1, 1, (rows, min(K, 32)))[spread] * 3.3e38
    if last:
        x[:, last:] *= 2.0 ** -125
    q, s = pack8(x.astype(np.float32))
    assert (s[big, 0] >= 246).all() and (s[0, 0] >= 247) and (not last or (s[:, -1] <= 2).all())
    b = r.standard_normal((rows, N)) * 2.0 ** small
    if large is not None:
        b[:, N // 2:] *= 2.0 ** (large - small)
    b = rounded(b, kind)
    qd, sd, bd = e.rows(q, "i8", 0), e.rows(s, "u8", 0), e.rows(b, kind, 0)
    G, ends = len(sizes), np.concatenate([[0], np.cumsum(sizes)])
    o, c = e.put(ends.astype(np.int64)), e.rows(np.full((G * K, N), 7.0), "f32", 0)
    Call(e, 0)(e.lib.gcn_gemm_grouped_q8, G, o.ptr, rows, N, K, qd.ptr, qd.ld, sd.ptr, sd.ld, bd.ptr, bd.ld,
               CODE[kind], c.ptr, c.ld, K * N)
    got = c.get().reshape(G, K, N)
    for g in range(G):
        rng = slice(ends[g], ends[g + 1])
        u, v = unpack8(q[rng], s[rng]), b[rng].astype(np.float64)
        want, mag = u.T @ v, np.abs(u).T @ np.abs(v)
        # a chain of sums; products below 2^-126 and their sums may be lost. Sums of magnitudes that fp32
        # does not hold may be infinities or NaN
        near = np.abs(got[g] - want) <= (sizes[g] + 8) * U * mag + sizes[g] * 2.0 ** -126
        bad = ~near & (mag < 3e38)
        assert not bad.any(), (sizes, K, N, kind, small, large, g, bad.sum(), np.argwhere(bad)[:3], got[g][bad][:3],
                               want[bad][:3])
