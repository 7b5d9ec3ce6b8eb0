"""The routed layer's operators on the GPU against the 64-bit references of routed_ref.py, and a layer made
of them."""

import ctypes

import numpy as np
import pytest

import routed_ref as ref
from gpu_util import dev, host, note

pytestmark = pytest.mark.gpu

KINDS = ("f32", "bf16")


@pytest.fixture(scope="module")
def G():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2411_16025_amd as pkg
    pkg.lib()
    return pkg


class Array:
    def __init__(self, flat, t, kind=None):
        self.flat, self.t, self.kind, self.ptr = flat, t, kind, ctypes.c_void_p(t.data_ptr())
        self.ld = max(t.stride(0), t.shape[1]) if t.dim() == 2 else 0

    def get(self):
        return host(self.t.float() if self.kind in KINDS else self.t)

    def check_margins(self):
        import torch
        before = self.flat.clone()
        self.t.fill_(5)
        fill = self.flat
        inside = torch.zeros_like(self.flat, dtype=torch.bool)
        torch.as_strided(inside, self.t.shape, self.t.stride(), self.t.storage_offset()).fill_(True)
        rest = fill[~inside]
        same = (rest == self.fill) | (rest.float().isnan() if rest.is_floating_point() else (rest == self.fill))
        assert bool(same.all()), "written between the rows"
        self.flat.copy_(before)


class Engine:
    """Memory of torch's, the library's entry points on the current stream."""

    def __init__(self, G):
        import torch
        self.lib, self.torch, self.kept = G.lib(), torch, []
        self.types = {"f32": torch.float32, "bf16": torch.bfloat16, "i8": torch.int8, "u8": torch.uint8}

    @property
    def stream(self):
        return ctypes.c_void_p(self.torch.cuda.current_stream().cuda_stream)

    def error(self):
        return self.lib.gcn_last_error().decode()

    def keep(self, a):
        self.kept.append(a)
        return a

    def put(self, a):
        t = dev(np.ascontiguousarray(a))
        return self.keep(Array(t, t))

    def new(self, shape, dtype):
        return self.put(np.full(shape, 77, dtype))

    def work(self, size):
        """With a margin of NaN bytes behind it (looked at by nobody: the kernels' CPU model does)."""
        t = self.torch.full((size,), 255, dtype=self.torch.uint8, device="cuda:0")
        assert t.data_ptr() % 256 == 0
        self.kept.append(t)
        return ctypes.c_void_p(t.data_ptr())

    def rows(self, x, kind, pad=0, shift=0, fill=np.nan):
        n, F = x.shape
        t = self.types[kind]
        if kind not in KINDS:
            fill = 77 if fill != fill else int(fill)
        flat = self.torch.full((shift + n * (F + pad) + 8,), fill, dtype=t, device="cuda:0")
        v = flat[shift:shift + n * (F + pad)].view(n, F + pad)[:, :F] if n else flat[:0].view(0, F)
        if n:
            v.copy_(dev(x).to(t))
        a = Array(flat, v, kind)
        if n == 0:
            a.ld = F
        a.fill = fill
        return self.keep(a)


@pytest.fixture()
def E(G):
    import torch
    e = Engine(G)
    yield e
    torch.cuda.synchronize()


def run(E, check, *args, **kw):
    note("%s %s %s" % (check, args, kw))
    getattr(ref, check)(E, *args, **kw)


# ---- positions by group ------------------------------------------------------------

@pytest.mark.parametrize("how", ["spread", "skew", "one", "none"])
@pytest.mark.parametrize("n,groups", [(0, 5), (1, 1), (1, 9), (64, 16), (1000, 3), (1025, 64), (100003, 17),
                                      (20000, 300), (4097, 2047), (4097, 2048), (70000, 50000), (5, 1 << 22),
                                      (3000, (1 << 22) + 5), (600001, 512), (600001, 2449029)])
def test_group_ids(E, n, groups, how):
    for memory in (0, 1):
        run(E, "check_group_ids", n, groups, how, memory=memory, seed=n + groups)


# tiles of 16,384 ids in one, two and three passes; of 4096 and 1024 ids in three
@pytest.mark.parametrize("how", ["spread", "skew", "one", "none"])
@pytest.mark.parametrize("n,groups", [((1 << 20) + 1, 37), ((1 << 20) + 777, 2047), ((1 << 20) + 777, 5000),
                                      ((1 << 20) + 777, (1 << 22) + 5), (5000003, 300), (3000001, 1 << 23),
                                      (1 << 20, (1 << 22) + 5), (1 << 18, 1 << 24), (20000, (1 << 25) + 1)])
def test_group_ids_of_many(E, n, groups, how):
    run(E, "check_group_ids", n, groups, how, memory=1, seed=n + groups)


@pytest.mark.parametrize("only", ["slot", "order"])
def test_group_ids_one_output(E, only):
    for groups in (9, 3000):
        run(E, "check_group_ids", 5000, groups, "none", only=only)


# ---- rows of a table ---------------------------------------------------------------

SHAPES = [(1, 1, 1), (3, 5, 2), (7, 8, 9), (40, 47, 11), (33, 100, 64), (1000, 33, 70), (129, 256, 300),
          (5, 264, 3), (3, 2049, 2), (2, 20001, 2), (5000, 64, 1000)]


@pytest.mark.parametrize("kt", KINDS)
@pytest.mark.parametrize("ky", KINDS)
@pytest.mark.parametrize("n,F,V", SHAPES + [(0, 4, 3), (40000, 128, 500)])
def test_embed_fwd(E, n, F, V, kt, ky):
    for pad, shift, per in ((0, 0, 1), (8, 0, 2), (3, 1, 7)):
        run(E, "check_embed_fwd", n, F, V, per=per, kt=kt, ky=ky, pad=pad, shift=shift, seed=n + F)


@pytest.mark.parametrize("kd", KINDS)
@pytest.mark.parametrize("kt", KINDS)
@pytest.mark.parametrize("n,F,V,how", [s + ("none",) for s in SHAPES] +
                         [(0, 4, 3, "spread"), (500, 9, 3, "skew"), (3000, 47, 30, "skew"), (700, 2049, 2, "one"),
                          (20000, 17, 1, "one"), (30000, 100, 4000, "skew"), (9000, 300, 20000, "spread"),
                          (300000, 12, 2, "spread")])
def test_embed_bwd(E, n, F, V, how, kd, kt):
    for i, (pad, shift) in enumerate(((0, 0), (3, 1))):
        run(E, "check_embed_bwd", n, F, V, how=how, kd=kd, kt=kt, pad=pad, shift=shift, add=bool(i), memory=i,
            seed=n + F)


@pytest.mark.parametrize("kt", KINDS)
@pytest.mark.parametrize("n,F,V", [(30, 7, 3000), (5, 100, 900), (40, 3, 2001), (1, 1, 9), (500, 47, 30000),
                                   (500, 47, 6000), (2000, 101, 20000)])
def test_embed_bwd_sparse(E, n, F, V, kt):
    """Most rows without a place, rows of dT beside each other, from an address of any element."""
    for shift in (0, 1, 3):
        run(E, "check_embed_bwd", n, F, V, how="skew", kt=kt, pad=-2, shift=shift, seed=n + F)


# ---- the router --------------------------------------------------------------------

ROUTES = [(1, 1, 1), (3, 2, 2), (70, 8, 3), (65, 9, 8), (500, 16, 2), (33, 47, 5), (400, 64, 8), (90, 100, 64),
          (210, 256, 4), (60, 257, 9), (70, 512, 8), (50, 513, 3), (40, 1024, 64), (0, 8, 2), (30001, 16, 4),
          (70000, 4, 2), (9000, 128, 8)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("how", ["plain", "ties", "closed", "far"])
@pytest.mark.parametrize("n,experts,k", ROUTES)
def test_route(E, n, experts, k, kind, how):
    for i, (normalize, masked) in enumerate(((False, True), (True, False), (True, True))):
        run(E, "check_route", n, experts, k, kind=kind, how=how, normalize=normalize, masked=masked, pad=3 * i,
            shift=i, memory=i & 1, loss=i != 1, seed=n + experts)


@pytest.mark.parametrize("normalize", [False, True])
def test_route_gradient_by_differences(G, normalize):
    """The gradient of sum(weights * g) + loss against differences of the 64-bit definition, whose choice and
    counts stay the same."""
    note("route differences")
    import torch
    r = np.random.default_rng(3)
    n, E, k, coef = 7, 12, 3, 0.5
    z = r.permuted(np.tile(np.arange(E) * 0.4, (n, 1)), axis=1).astype(np.float32)
    g = r.standard_normal((n, k)).astype(np.float32)
    zd = dev(z)
    ex, w, counts, loss = G.gcn_route_fwd(zd, k, coef=coef, normalize=normalize)
    dz = host(G.gcn_route_bwd(zd, ex, w, counts, dweights=dev(g), coef=coef, normalize=normalize)).astype(np.float64)
    at, c = host(ex).astype(np.int64), host(counts)

    def total(z):
        p, _ = ref.softmax(z)
        v = np.take_along_axis(p, at, 1)
        if normalize:
            v = v / v.sum(1, keepdims=True)
        return (v * g).sum() + coef * E * (c[:E] / c[:E].sum() * p.sum(0) / c[E]).sum()
    h = 1e-5
    for t in range(n):
        for e in range(E):
            up, down = z.astype(np.float64), z.astype(np.float64)
            up[t, e] += h
            down[t, e] -= h
            d = (total(up) - total(down)) / (2 * h)
            # the differences are off by h^2 / 6 of a third derivative of a few units and by the roundings of
            # 64-bit sums over 2 h; dz itself by some 60 U of numbers of order 1
            assert abs(d - dz[t, e]) <= 1e-9 + 1e-10 + 200 * ref.U, (t, e, d, dz[t, e])
    assert torch.isfinite(loss)


def test_route_special_values(G):
    note("route special values")
    import torch
    z = torch.zeros((6, 5), device="cuda:0")
    z[0, 2] = float("nan")
    z[1] = float("-inf")
    z[2, 3] = float("inf")
    z[3] = torch.tensor([1.0, float("-inf"), 1.0, float("nan"), 1.0])
    z[4, :] = float("nan")
    z[5] = torch.tensor([0.0, 1.0, 1.0, 0.5, -0.0])
    for normalize in (False, True):
        ex, w, c, loss = G.gcn_route_fwd(z, 4, coef=1.0, normalize=normalize)
        ex, w = host(ex), host(w)
        assert ex.tolist() == [[0, 1, 3, 4], [-1] * 4, [3, 0, 1, 2], [0, 2, 4, -1], [-1] * 4, [1, 2, 3, 0]]
        assert np.isnan(w[[0, 2]]).all() and np.isnan(w[3, :3]).all() and (w[1] == 0).all() and w[3, 3] == 0
        assert (w[4] == 0).all() and np.isfinite(w[5]).all()
        assert np.isnan(host(loss)) and host(c).tolist() == [4, 3, 3, 3, 2, 4]
        dz = host(G.gcn_route_bwd(z, dev(ex), dev(w), c, coef=1.0, normalize=normalize))
        assert (dz[[1, 4]] == 0).all() and np.isnan(dz[[0, 2]]).any(1).all() and np.isfinite(dz[5]).all()
    ex, w, c, loss = G.gcn_route_fwd(z[1:2], 2, coef=1.0)
    assert host(c).tolist() == [0] * 6 and float(loss) == 0.0


# ---- back from the groups' order ------------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,k,F,rows", [(1, 1, 1, 1), (3, 2, 5, 6), (200, 8, 47, 1600), (90, 3, 64, 200),
                                        (5, 1, 100, 9), (4, 5, 264, 0), (30, 2, 1000, 60), (20, 9, 2049, 180),
                                        (3000, 4, 16, 12000), (0, 2, 8, 3), (30, 2, 4200, 50), (3, 2, 20001, 6),
                                        (999, 8, 1024, 9000), (500, 64, 24, 40000)])
def test_combine(E, n, k, F, rows, kind):
    for i, (pad, shift) in enumerate(((0, 0), (8, 0), (3, 1))):
        run(E, "check_combine", n, k, F, rows, kind=kind, weighted=i != 1, pad=pad, shift=shift, in_place=i == 2,
            seed=n + F)


# ---- rows in 8 bits ----------------------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("how", ["plain", "sizes", "edges", "special"])
@pytest.mark.parametrize("n,F", [(1, 1), (3, 7), (5, 32), (9, 33), (40, 47), (200, 100), (700, 256), (3, 2049),
                                 (5, 4100), (0, 8), (2, 20001), (3000, 64)])
def test_pack8(E, n, F, kind, how):
    for pad, shift in ((0, 0), (8, 0), (3, 1)):
        run(E, "check_pack8", n, F, kind=kind, how=how, pad=pad, shift=shift, seed=n + F)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("memory", [0, 1])
@pytest.mark.parametrize("sizes,K,N", [([1], 1, 1), ([5], 3, 7), ([40, 0, 3], 33, 65), ([300], 100, 47),
                                       ([130, 700], 64, 64), ([20] * 30, 40, 24), ([0, 0], 5, 5),
                                       ([900, 0, 1], 130, 129), ([513], 256, 264), ([5000, 300], 512, 1000),
                                       ([3000, 0, 2500], 264, 520), ([20000], 8, 8), ([9], 2000, 600),
                                       ([10] * 1100, 32, 16), ([4000, 1], 100, 2048), ([700, 0, 90], 136, 520),
                                       ([33, 1] * 3, 16, 8), ([257], 300, 140), ([70, 3], 17, 257),
                                       ([30000, 5000], 100, 256), ([3000] * 9, 260, 130)])
def test_grad8(E, sizes, K, N, kind, memory):
    for pad, whole in ((0, True), (8, False), (3, True)):
        run(E, "check_grad8", sizes, K, N, kind=kind, before=pad, after=memory, pad=pad, memory=memory, whole=whole,
            seed=K + N)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,K,N", [(40, 64, 8), (100, 150, 20), (300, 260, 264), (9, 40, 7), (5000, 300, 520)])
def test_grad8_special(E, rows, K, N, kind):
    run(E, "check_grad8_special", rows, K, N, kind=kind, seed=K)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("sizes,K,N", [([12], 7, 3), ([40], 64, 9), ([40], 64, 8), ([700], 40, 16), ([600], 33, 20),
                                       ([300], 260, 264), ([300], 256, 136), ([40, 0, 30], 150, 20),
                                       ([2000, 900], 512, 1000), ([3000], 100, 47), ([2000], 261, 257)])
def test_grad8_scales(E, sizes, K, N, kind):
    """Scale bytes from 1 to 248, which packing gives to finite values."""
    for how in (dict(), dict(small=-100), dict(large=100)):
        run(E, "check_grad8_scales", sizes, K, N, kind=kind, seed=K, **how)


# ---- a layer --------------------------------------------------------------------------

def test_layer(G):
    """A training step of a routed layer out of the calls, against its 64-bit form on what the calls chose."""
    note("routed layer")
    import torch
    r = np.random.default_rng(9)
    n, V, F, H, E, k, coef = 700, 90, 100, 72, 6, 2, 0.3
    ids = r.integers(-1, V, n).astype(np.int32)
    table = r.standard_normal((V, F)).astype(np.float32)
    Wr = (r.standard_normal((F, E)) / 10).astype(np.float32)
    W = (r.standard_normal((E, F, H)) / 10).astype(np.float32)
    dy = r.standard_normal((n, H)).astype(np.float32)
    mask = (r.random(n) < 0.9).astype(np.uint8)
    d = {nm: dev(v) for nm, v in dict(ids=ids, table=table, Wr=Wr, W=W, dy=dy, mask=mask).items()}
    x = G.gcn_embed_fwd(d["table"], d["ids"], scale=1.5)
    z = G.gcn_gemm_f32(G.GCN_GEMM_NN, x, d["Wr"])
    experts, w, counts, loss = G.gcn_route_fwd(z, k, mask=d["mask"], coef=coef, normalize=True)
    offsets, order, slot = G.gcn_group_ids(experts.view(-1), E)
    slot = slot.view(n, k)
    xs = G.gcn_embed_fwd(x, order, per=k)
    Q, S = G.gcn_pack8(xs)
    h = G.gcn_gemm_grouped(G.GCN_GEMM_NN, offsets, xs, d["W"])
    y = G.gcn_combine_fwd(h, slot, w)
    # backward
    dh, dw = G.gcn_combine_bwd(h, slot, w, d["dy"], dZ=h)
    dW = G.gcn_gemm_grouped_q8(offsets, Q, S, dh)
    dxs = G.gcn_gemm_grouped(G.GCN_GEMM_NT, offsets, dh, d["W"])
    dx = G.gcn_combine_fwd(dxs, slot)
    dz = G.gcn_route_bwd(z, experts, w, counts, dweights=dw, coef=coef, normalize=True)
    dx += G.gcn_gemm_f32(G.GCN_GEMM_NT, dz, d["Wr"])
    dWr = G.gcn_gemm_f32(G.GCN_GEMM_TN, x, dz)
    by_id, places, _ = G.gcn_group_ids(d["ids"], V, slots=False)
    dT = G.gcn_embed_bwd(dx, by_id, places, scale=1.5)
    torch.cuda.synchronize()

    # 64 bits
    ex = host(experts).astype(np.int64)
    real = ids >= 0
    X = np.where(real[:, None], 1.5 * table[np.maximum(ids, 0)].astype(np.float64), 0)
    Z = X @ Wr
    p, _ = ref.softmax(Z)
    on = ex >= 0
    assert np.array_equal(on.all(1), mask == 1)
    pk = np.where(on, np.take_along_axis(p, np.maximum(ex, 0), 1), 0)
    s = np.where(on.any(1), pk.sum(1), 1)[:, None]
    wk = pk / s
    H_all = np.einsum("nf,efh->neh", X, W.astype(np.float64))
    Hk = np.take_along_axis(H_all, np.maximum(ex, 0)[:, :, None], 1) * on[:, :, None]
    Y = (wk[:, :, None] * Hk).sum(1)
    near = lambda got, want, rel, nm: ref_near(got, want, rel, nm)  # noqa: E731
    # each value passes some thousand roundings of fp32 at most, along sums of F, H or n terms: 1e-4 of the
    # largest value holds them with a margin of ten; the 8-bit rows are off by 1 / 254 of their 32 columns'
    # largest, independently: sums over the rows by less than 1 / 254 of the sum of magnitudes
    near(y, Y, 1e-4, "y")
    dwk = np.einsum("nh,nkh->nk", dy.astype(np.float64), Hk)
    near(dw, dwk, 1e-4, "dw")
    dZk = np.where(on, wk * (dwk - (dwk * wk).sum(1, keepdims=True)), 0)
    dZ = np.zeros((n, E))
    np.add.at(dZ, (np.arange(n)[:, None], np.maximum(ex, 0)), dZk)
    c = host(counts)
    a = coef * E * c[:E] / (c[:E].sum() * c[E])
    pm = np.where(on[:, :1], p, 0)
    dZ += pm * (a - (pm * a).sum(1, keepdims=True))
    near(dz, dZ, 1e-4, "dz")
    assert abs(float(loss) - coef * E * (c[:E] / c[:E].sum() * pm.sum(0) / c[E]).sum()) < 1e-5
    dXk = np.zeros((n, F))
    dWw, mag = np.zeros((E, F, H)), np.zeros((E, F, H))
    for i in range(k):
        for e in range(E):
            t = np.nonzero(ex[:, i] == e)[0]
            dh_ = wk[t, i][:, None] * dy[t]
            dXk[t] += dh_ @ W[e].T
            dWw[e] += X[t].T @ dh_
            top = np.abs(X[t]).max(1, keepdims=True)
            mag[e] += (np.ones((1, F)) * top).T @ np.abs(dh_)
    dXk += dZ @ Wr.T
    near(dWr, X.T @ dZ, 1e-4, "dWr")
    assert (np.abs(host(dW) - dWw) <= mag / 127 + 1e-4 * np.abs(dWw).max()).all()
    dTt = np.zeros((V, F))
    np.add.at(dTt, ids[real], 1.5 * dXk[real])
    near(dT, dTt, 1e-4, "dT")


def ref_near(got, want, rel, what):
    err = np.abs(host(got) - want).max()
    assert err <= rel * np.abs(want).max(), (what, err, np.abs(want).max())
