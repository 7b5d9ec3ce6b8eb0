"""64-bit references of the typed layer's operators (host, numpy)."""

import numpy as np

U = 2.0 ** -24         # half a step of fp32
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}  # half a step of a type, relative

M0, M1, W0, W1 = 0xD2511F53, 0xCD9E8D57, 0x9E3779B9, 0xBB67AE85
LOW = np.uint64(0xFFFFFFFF)


def philox(counter, key, rounds=7):
    """Philox4x32 of counters [..., 4] under a key (k0, k1): the definition, round by round."""
    c = [np.asarray(counter[..., i], np.uint64) for i in range(4)]
    k0, k1 = key
    s = np.uint64(32)
    for _ in range(rounds):
        a, b = c[0] * np.uint64(M0), c[2] * np.uint64(M1)
        c = [(b >> s) ^ c[1] ^ np.uint64(k0), b & LOW, (a >> s) ^ c[3] ^ np.uint64(k1), a & LOW]
        k0, k1 = (k0 + W0) & 0xFFFFFFFF, (k1 + W1) & 0xFFFFFFFF
    return np.stack(c, -1)


def words(n, F, seed, call, row0=0):
    cols = (F + 3) // 4
    c = np.zeros((n, cols, 4), np.uint64)
    c[..., 0] = np.arange(cols, dtype=np.uint64)
    c[..., 1] = (row0 + np.arange(n, dtype=np.uint64))[:, None]
    c[..., 2] = call & 0xFFFFFFFF
    c[..., 3] = (call >> 32) & 0xFFFFFFFF
    return philox(c, (seed & 0xFFFFFFFF, seed >> 32)).reshape(n, -1)[:, :F]


def kept(n, F, p, seed, call=0, row0=0):
    return words(n, F, seed, call, row0) >= np.uint64(int(p * 4294967296.0))


def factor(n, F, p, seed, call=0, row0=0):
    """What dropout multiplies by."""
    return kept(n, F, p, seed, call, row0) / (1.0 - p)


def norm(x, eps):
    """(H, rstd) of the rows."""
    x = np.asarray(x, np.float64)
    d = x - x.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt((d * d).mean(1, keepdims=True) + eps)
    return d * rstd, rstd


def norm_fwd(x, gamma, beta, eps, drop=1.0):
    h, _ = norm(x, eps)
    return (h * gamma + beta) * drop


def norm_fwd_bound(x, gamma, beta, eps, drop, kind):
    """h: x - mean in two differences, rstd and their product rounded to fp32, 4 U; its
    product with gamma and the sum 1 U of each; the factor 2 U: 8 U of |h gamma| + |beta|
    with a margin, and half a step of the type."""
    h, _ = norm(x, eps)
    y = (np.abs(h * gamma) + np.abs(beta)) * drop
    return 8 * U * y + (HALF[kind] if kind != "f32" else 0.0) * np.abs((h * gamma + beta) * drop)


def norm_bwd(x, dy, gamma, eps, drop=1.0):
    h, rstd = norm(x, eps)
    g = np.asarray(dy, np.float64) * drop
    t = g * gamma
    dx = rstd * (t - t.mean(1, keepdims=True) - h * (t * h).mean(1, keepdims=True))
    return dx, (g * h).sum(0), g.sum(0)


def norm_bwd_bound(x, dy, gamma, eps, drop, kind):
    """Worst cases of the roundings: g 2 U, t 3 U, h 4 U; a mean over F in fp32 adds D U of the
    mean of magnitudes, D the longest chain of additions (at most 64 elements of a lane,
    or F / 256 where a workgroup walks the row, and 16 steps of the joins); the
    differences and the product with rstd 1 U each."""
    n, F = x.shape
    D = 80 + F / 256
    h, rstd = norm(x, eps)
    g = np.asarray(dy, np.float64) * drop
    t = g * gamma
    at, ath = np.abs(t).mean(1, keepdims=True), np.abs(t * h).mean(1, keepdims=True)
    dx = rstd * U * (8 * np.abs(t) + (D + 8) * at + (D + 16) * np.abs(h) * ath)
    ref = norm_bwd(x, dy, gamma, eps, drop)[0]
    half = HALF[kind] if kind != "f32" else 0.0
    return (dx + half * np.abs(ref), (n + 16) * U * np.abs(g * h).sum(0),
            (n + 16) * U * np.abs(g).sum(0))


def grouped(op, ends, a, b):
    """(result, sum of magnitudes) of one product per group; rows of no group 0."""
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    G = len(ends) - 1
    if op == 2:
        out = np.zeros((2, G, a.shape[1], b.shape[1]))
    else:
        out = np.zeros((2, a.shape[0], b.shape[2 if op == 0 else 1]))
    sides = ((a, b), (np.abs(a), np.abs(b)))
    for g in range(G):
        r = slice(ends[g], ends[g + 1])
        for i, (x, y) in enumerate(sides):
            if ends[g] == ends[g + 1]:
                continue
            if op == 0:
                out[i][r] = x[r] @ y[g]
            elif op == 1:
                out[i][r] = x[r] @ y[g].T
            else:
                out[i][g] = x[r].T @ y[r]
    return out[0], out[1]


def grouped_bound(ref, mag, depth, kind_out):
    """Sums of `depth` products in fp32: at most depth U of the magnitudes, and the products
    themselves 8 U; half a step of the output's type."""
    half = HALF[kind_out] if kind_out != "f32" else 0.0
    return (depth + 8) * U * mag + half * np.abs(ref)
