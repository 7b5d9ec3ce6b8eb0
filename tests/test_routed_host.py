"""The routed layer's calls on the host: refusals (nothing is launched)."""

import ctypes

import numpy as np
import pytest

import routed_ref as ref

EINVAL, ERANGE = 1, 2
A, B, C = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000), ctypes.c_void_p(0x3000)
ODD = ctypes.c_void_p(0x1010)


@pytest.fixture(scope="module")
def L():
    import paper_2411_16025_amd as pkg
    return pkg.lib()


def refused(f, defaults, cases, status=EINVAL):
    for kw in cases:
        assert f(*{**defaults, **kw}.values()) == status, kw


def test_group_ids_refusals(L):
    d = dict(n=4, ids=A, groups=3, offsets=B, order=C, slot=C, work=None, size=None, stream=None)
    some = ctypes.byref(ctypes.c_int64(1 << 30))
    refused(L.gcn_group_ids, d, [dict(n=-1), dict(groups=0), dict(groups=-5), dict(ids=None), dict(offsets=None),
                                 dict(work=A), dict(work=ODD, size=some), dict(order=A), dict(slot=A)])
    refused(L.gcn_group_ids, d, [dict(n=1 << 31), dict(groups=(1 << 30) + 1)], ERANGE)
    size = ctypes.c_int64(-1)
    ask = dict(size=ctypes.byref(size))
    # two lists of ids with their positions and one of ids, 20 bytes an id; 2048 counts of 4 bytes for every
    # 4096 ids (1024 of few), 2 bytes an id
    for n, groups, most in ((5000, 3, 1 << 14), (1 << 20, 16, 1 << 16), (1 << 20, 1 << 22, 22 << 20),
                            ((1 << 31) - 1, 1 << 30, (22 << 31) + (1 << 20))):
        assert L.gcn_group_ids(*{**d, **ask, "n": n, "groups": groups}.values()) == 0
        assert 0 < size.value <= most, (n, groups, size.value)
    less = ctypes.byref(ctypes.c_int64(256))
    refused(L.gcn_group_ids, d, [dict(n=100000, work=A, size=less)])


def at(address):
    return ctypes.c_void_p(address)


def test_group_ids_refuses_arrays_over_each_other(L):
    """Wherever one begins in the other (nothing is launched); the question for the scratch memory's size
    looks at no array."""
    n, G = 1000, 99
    d = dict(n=n, ids=at(0x10000), groups=G, offsets=at(0x20000), order=at(0x30000), slot=at(0x40000), work=None, size=None,
             stream=None)
    first = dict(ids=0x10000, offsets=0x20000, order=0x30000, slot=0x40000)
    size = dict(ids=4 * n, offsets=8 * (G + 1), order=4 * n, slot=4 * n)
    for a in first:
        for b in first:
            if a != b:
                refused(L.gcn_group_ids, d, [{a: at(first[b])}, {a: at(first[b] + size[b] - 8)},
                                             {a: at(first[b] - size[a] + 8)}])
    want = ctypes.c_int64(-1)
    assert L.gcn_group_ids(*{**d, "groups": 5000, "slot": d["order"], "size": ctypes.byref(want)}.values()) == 0
    assert want.value > 0


X, Y, Z, W, V = (0x100000 * (i + 1) for i in range(5))


def both_ways(f, d, out, at_in, out_bytes, in_bytes):
    """Output `out` refused over the input at `at_in`, from either end (nothing is launched)."""
    refused(f, d, [{out: at(at_in + in_bytes - 2)}, {out: at(at_in - out_bytes + 2)}, {out: at(at_in + 2)}])


def test_matrices_over_each_other_are_refused(L):
    n, F, V_ = 50, 40, 60
    d = dict(n=n, F=F, V=V_, ids=at(X), per=1, T=at(Y), ldt=F + 3, dt=0, scale=1.0, Y=at(Z), ldy=F, dy=1, stream=None)
    t = 4 * ((V_ - 1) * (F + 3) + F)
    both_ways(L.gcn_embed_fwd, d, "Y", Y, 2 * n * F, t)
    both_ways(L.gcn_embed_fwd, d, "Y", X, 2 * n * F, 4 * n)
    # rows between the other's rows, of the same stride, that reach into the next one or begin in the last one
    wide = {**d, "ldt": 2 * F, "ldy": 4 * F}
    refused(L.gcn_embed_fwd, wide, [dict(Y=at(Y + 8 * F - 2)), dict(Y=at(Y + 4 * F - 2)), dict(Y=at(Y - 2 * F + 2))])
    # of another stride, whose first rows lie between them
    refused(L.gcn_embed_fwd, wide, [dict(Y=at(Y + 4 * F), ldy=4 * F + 2), dict(Y=at(Y + 4 * F), ldy=3 * F)])
    d = dict(n=n, F=F, V=V_, offsets=at(X), order=at(W), dY=at(Y), lddy=F, dt=1, scale=1.0, dT=at(Z), lddt=F, dtt=0, flags=0,
             work=None, size=None, stream=None)
    for a, b in ((Y, 2 * n * F), (X, 8 * (V_ + 1)), (W, 4 * n)):
        both_ways(L.gcn_embed_bwd, d, "dT", a, 4 * V_ * F, b)
    E, k = 20, 3
    d = dict(n=n, E=E, z=at(X), ldz=E, dt=0, k=k, flags=0, mask=at(X + 0x8000), coef=0.1, experts=at(Y), weights=at(Z),
             counts=at(W), loss=at(V), work=None, size=None, stream=None)
    size = dict(z=4 * n * E, mask=n, experts=4 * n * k, weights=4 * n * k, counts=8 * (E + 1), loss=4)
    for out in ("experts", "weights", "counts", "loss"):
        for other in size:
            if other != out:
                a = d[other].value
                refused(L.gcn_route_fwd, d, [{out: at(a)}, {out: at(a + size[other] - 1)}, {out: at(a - size[out] + 1)}])
    b = dict(n=n, E=E, z=at(X), ldz=E, dt=0, k=k, flags=0, experts=at(Y), weights=at(Z), counts=at(W), coef=0.1, dw=at(V),
             dloss=None, dz=at(V + 0x8000), ldd=E, stream=None)
    for a, m in ((X, 4 * n * E), (Y, 4 * n * k), (Z, 4 * n * k), (W, 8 * (E + 1)), (V, 4 * n * k)):
        both_ways(L.gcn_route_bwd, b, "dz", a, 4 * n * E, m)
    rows = 200
    d = dict(n=n, k=k, F=F, Z=at(X), rows=rows, ldz=F, dt=1, slot=at(Y), w=at(Z), Y=at(W), ldy=F, stream=None)
    for a, m in ((X, 2 * rows * F), (Y, 4 * n * k), (Z, 4 * n * k)):
        both_ways(L.gcn_combine_fwd, d, "Y", a, 2 * n * F, m)
    b = dict(n=n, k=k, F=F, Z=at(X), rows=rows, ldz=F, dt=1, slot=at(Y), w=at(Z), dY=at(W), lddy=F, dZ=at(V), lddz=F,
             dw=at(V + 0x8000), stream=None)
    for a, m in ((X, 2 * rows * F), (Y, 4 * n * k), (Z, 4 * n * k), (W, 2 * n * F), (V + 0x8000, 4 * n * k)):
        both_ways(L.gcn_combine_bwd, b, "dZ", a, 2 * rows * F, m)
    for a, m in ((X, 2 * rows * F), (Y, 4 * n * k), (W, 2 * n * F)):
        both_ways(L.gcn_combine_bwd, b, "dw", a, 4 * n * k, m)
    d = dict(n=n, F=F, X=at(X), ldx=F, dt=0, Q=at(Y), ldq=F, S=at(Z), lds=2, stream=None)
    both_ways(L.gcn_pack8, d, "Q", X, n * F, 4 * n * F)
    both_ways(L.gcn_pack8, d, "S", X, n * 2, 4 * n * F)
    both_ways(L.gcn_pack8, d, "S", Y, n * 2, n * F)
    refused(L.gcn_pack8, d, [dict(Q=at(X)), dict(S=at(Y)), dict(ldq=F + 2, lds=F + 2, S=at(Y + F + 1))])
    u = dict(n=n, F=F, Q=at(Y), ldq=F, S=at(Z), lds=2, Y=at(X), ldy=F, dt=0, stream=None)
    both_ways(L.gcn_unpack8, u, "Y", Y, 4 * n * F, n * F)
    both_ways(L.gcn_unpack8, u, "Y", Z, 4 * n * F, n * 2)
    G, N, K = 2, 8, 40
    d = dict(G=G, off=at(X), rows=n, N=N, K=K, Q=at(Y), ldq=K, S=at(Z), lds=2, B=at(W), ldb=N, dt=0, C=at(V), ldc=N, sw=K * N,
             work=None, size=None, stream=None)
    for a, m in ((X, 8 * (G + 1)), (Y, n * K), (Z, n * 2), (W, 4 * n * N)):
        both_ways(L.gcn_gemm_grouped_q8, d, "C", a, 4 * G * K * N, m)


def test_embed_refusals(L):
    d = dict(n=4, F=8, V=5, ids=A, per=1, T=B, ldt=8, dt=0, scale=1.0, Y=C, ldy=8, dy=0, stream=None)
    refused(L.gcn_embed_fwd, d, [dict(n=-1), dict(F=0), dict(F=(1 << 30) + 1), dict(V=0), dict(V=-1), dict(ids=None),
                                 dict(per=0), dict(per=1 << 31), dict(T=None), dict(Y=None), dict(Y=B), dict(ldt=7),
                                 dict(ldy=7), dict(dt=2), dict(dy=-1), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(scale=1e300)])
    refused(L.gcn_embed_fwd, d, [dict(n=1 << 31), dict(V=1 << 31)], ERANGE)
    assert L.gcn_embed_fwd(*{**d, "n": 0, "ids": None, "Y": None}.values()) == 0
    d = dict(n=4, F=8, V=5, offsets=A, order=A, dY=B, lddy=8, dt=0, scale=1.0, dT=C, lddt=8, dtt=1, flags=0, work=None,
             size=None, stream=None)
    refused(L.gcn_embed_bwd, d, [dict(n=-1), dict(F=0), dict(V=0), dict(offsets=None), dict(order=None), dict(dY=None),
                                 dict(dT=None), dict(dT=B), dict(lddy=7), dict(lddt=7), dict(dt=3), dict(dtt=2),
                                 dict(flags=2), dict(scale=float("nan")), dict(work=A),
                                 dict(work=ODD, size=ctypes.byref(ctypes.c_int64(1 << 40)))])
    refused(L.gcn_embed_bwd, d, [dict(n=1 << 31), dict(V=(1 << 30) + 1)], ERANGE)
    assert L.gcn_embed_bwd(*{**d, "n": 0, "flags": 1, "order": None, "dY": None}.values()) == 0
    size = ctypes.c_int64(-1)
    big = dict(n=1 << 17, F=1000, lddy=1000, lddt=1000, V=50000)
    assert L.gcn_embed_bwd(*{**d, **big, "size": ctypes.byref(size)}.values()) == 0
    assert 0 < size.value <= (1 << 17) * 1000 * 4 // 16
    less = ctypes.byref(ctypes.c_int64(size.value - 256))
    refused(L.gcn_embed_bwd, {**d, **big}, [dict(work=A, size=less)])


def test_route_refusals(L):
    d = dict(n=4, E=8, z=A, ldz=8, dt=0, k=2, flags=0, mask=None, coef=0.1, experts=B, weights=B, counts=B, loss=B,
             work=None, size=None, stream=None)
    bad = [dict(n=-1), dict(E=0), dict(E=-1), dict(E=1025, ldz=1025), dict(k=0), dict(k=9), dict(E=100, ldz=100, k=65),
           dict(flags=2), dict(dt=2), dict(coef=float("nan")), dict(ldz=7), dict(z=None), dict(experts=None),
           dict(weights=None)]
    refused(L.gcn_route_fwd, d, bad + [dict(counts=None), dict(work=A)])
    refused(L.gcn_route_fwd, d, [dict(n=1 << 31), dict(n=1 << 30)], ERANGE)
    b = dict(n=4, E=8, z=A, ldz=8, dt=0, k=2, flags=0, experts=B, weights=B, counts=B, coef=0.1, dw=B, dloss=None, dz=C,
             ldd=8, stream=None)
    refused(L.gcn_route_bwd, b, bad + [dict(dz=None), dict(ldd=7), dict(dz=A, ldd=9), dict(counts=None)])
    refused(L.gcn_route_bwd, b, [dict(n=1 << 30)], ERANGE)
    assert L.gcn_route_bwd(*{**b, "n": 0, "z": None}.values()) == 0


def test_combine_refusals(L):
    d = dict(n=4, k=2, F=8, Z=A, rows=8, ldz=8, dt=0, slot=B, w=B, Y=C, ldy=8, stream=None)
    bad = [dict(n=-1), dict(k=0), dict(k=65537), dict(F=0), dict(rows=-1), dict(Z=None), dict(ldz=7), dict(dt=2),
           dict(slot=None)]
    refused(L.gcn_combine_fwd, d, bad + [dict(Y=None), dict(Y=A), dict(ldy=7)])
    refused(L.gcn_combine_fwd, d, [dict(n=1 << 31), dict(rows=1 << 31)], ERANGE)
    assert L.gcn_combine_fwd(*{**d, "n": 0, "Y": None}.values()) == 0
    b = dict(n=4, k=2, F=8, Z=A, rows=8, ldz=8, dt=0, slot=B, w=B, dY=C, lddy=8, dZ=ctypes.c_void_p(0x4000), lddz=8, dw=B,
             stream=None)
    refused(L.gcn_combine_bwd, b, bad + [dict(dY=None), dict(lddy=7), dict(lddz=7), dict(dZ=C), dict(dY=A),
                                         dict(dZ=A, lddz=9), dict(dZ=None, dw=None)])
    assert L.gcn_combine_bwd(*{**b, "n": 0, "dY": None}.values()) == 0


def test_pack8_refusals(L):
    d = dict(n=4, F=40, X=A, ldx=40, dt=0, Q=B, ldq=40, S=C, lds=2, stream=None)
    bad = [dict(n=-1), dict(F=0), dict(dt=2), dict(Q=None), dict(ldq=39), dict(S=None), dict(lds=1)]
    refused(L.gcn_pack8, d, bad + [dict(X=None), dict(ldx=39)])
    refused(L.gcn_pack8, d, [dict(n=1 << 31)], ERANGE)
    assert L.gcn_pack8(*{**d, "n": 0, "X": None, "Q": None}.values()) == 0
    u = dict(n=4, F=40, Q=B, ldq=40, S=C, lds=2, Y=A, ldy=40, dt=0, stream=None)
    refused(L.gcn_unpack8, u, bad + [dict(Y=None), dict(ldy=39)])


def test_grad8_refusals(L):
    d = dict(G=2, off=A, rows=4, N=8, K=40, Q=A, ldq=40, S=A, lds=2, B=B, ldb=8, dt=0, C=C, ldc=8, sw=320, work=None,
             size=None, stream=None)
    f = L.gcn_gemm_grouped_q8
    refused(f, d, [dict(G=0), dict(G=65536), dict(rows=-1), dict(N=0), dict(K=0), dict(N=1 << 24), dict(K=1 << 24),
                   dict(dt=2), dict(off=None), dict(Q=None), dict(S=None), dict(B=None), dict(C=None), dict(ldq=39),
                   dict(lds=1), dict(ldb=7), dict(ldc=7), dict(sw=319), dict(G=1, sw=-1), dict(ldq=1 << 41),
                   dict(work=A), dict(work=ODD, size=ctypes.byref(ctypes.c_int64(1 << 30)))])
    refused(f, d, [dict(rows=1 << 31)], ERANGE)
    refused(f, d, [dict(K=1 << 23, ldq=1 << 23, lds=1 << 18, N=1 << 23, ldb=1 << 23, ldc=1 << 23, sw=1 << 46)], ERANGE)
    size = ctypes.c_int64(-1)
    big = dict(rows=500000, N=256, K=256, ldq=256, lds=8, ldb=256, ldc=256, sw=65536)
    assert f(*{**d, **big, "size": ctypes.byref(size)}.values()) == 0
    assert 0 < size.value <= 134e6 and size.value % (256 * 256 * 4) == 0
    less = ctypes.byref(ctypes.c_int64(size.value - 256))
    refused(f, {**d, **big}, [dict(work=A, size=less)])


def test_reference_of_packed_rows():
    """The reference itself: every value is within half a unit, units are the least that do, and the codes'
    values are exact in bf16."""
    r = np.random.default_rng(1)
    x = ref.some_rows(r, 200, 100, "f32", "sizes").astype(np.float64)
    q, s = ref.pack8(x)
    unit = np.repeat(2.0 ** (s.astype(np.float64) - 127), 32, 1)[:, :100]
    v = ref.unpack8(q, s)
    assert (np.abs(v - x) <= unit / 2).all()
    top = np.abs(x)
    for b in range(4):
        c = slice(32 * b, 32 * b + 32)
        u = unit[:, c.start]
        m = top[:, c].max(1)
        assert (m <= 127 * u).all() and ((m > 127 * u / 2) | (s[:, b] == 1)).all()
    assert np.array_equal(ref.bf16_round(v.astype(np.float32)).astype(np.float64), v)
