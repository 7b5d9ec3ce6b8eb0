"""The typed layer's calls on the host: refusals (nothing is launched), and the mask's
reference against the generator's published answers."""

import ctypes
import math

import numpy as np
import pytest

import typed_ref as ref

EINVAL, ERANGE = 1, 2


@pytest.fixture(scope="module")
def L():
    import paper_2411_16025_amd as pkg
    return pkg.lib()


FAKE = ctypes.c_void_p(0x1000)


def spec(p=0.5, seed=1, call=0, row0=0):
    import paper_2411_16025_amd as pkg
    return pkg.Dropout(p, seed, call, row0)._ref()


@pytest.mark.parametrize("rounds,want", [
    (7, (0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48)),
    (10, (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8))])
def test_reference_generator(rounds, want):
    got = ref.philox(np.zeros((1, 4), np.uint64), (0, 0), rounds)[0]
    assert tuple(int(v) for v in got) == want


def test_reference_mask_share():
    """The share of kept elements lies within 5 standard deviations of 1 - p, and masks of
    neighbouring rows, calls and seeds are uncorrelated to that accuracy."""
    n, F = 512, 256
    for p in (0.1, 0.5, 0.9):
        sd = math.sqrt(p * (1 - p) / (n * F))
        k = [ref.kept(n, F, p, 7), ref.kept(n, F, p, 8), ref.kept(n, F, p, 7, call=1),
             ref.kept(n, F, p, 7, row0=1)]
        for m in k:
            assert abs(m.mean() - (1 - p)) < 5 * sd
        for m in k[1:]:
            c = ((k[0] - (1 - p)) * (m - (1 - p))).mean() / (p * (1 - p))
            assert abs(c) < 5 / math.sqrt(n * F)
    assert np.array_equal(ref.kept(8, 5, 0.5, 7, row0=3), ref.kept(11, 5, 0.5, 7)[3:])


def test_dropout_refusals(L):
    f = L.gcn_dropout
    ok = (4, 8, FAKE, 8, 0)
    assert f(-1, 8, FAKE, 8, 0, spec(), FAKE, 8, None) == EINVAL
    assert f(4, 0, FAKE, 8, 0, spec(), FAKE, 8, None) == EINVAL
    assert f(4, (1 << 30) + 1, FAKE, 1 << 31, 0, spec(), FAKE, 1 << 31, None) == EINVAL
    assert f(4, 8, FAKE, 8, 2, spec(), FAKE, 8, None) == EINVAL   # unknown dtype
    assert f(1 << 31, 8, FAKE, 8, 0, spec(), FAKE, 8, None) == ERANGE
    assert f(*ok, None, FAKE, 8, None) == EINVAL
    for p in (-0.1, 1.0, 1.5, float("nan")):
        assert f(*ok, spec(p), FAKE, 8, None) == EINVAL
    assert f(*ok, spec(row0=-1), FAKE, 8, None) == EINVAL
    assert f(*ok, spec(row0=(1 << 32) - 3), FAKE, 8, None) == ERANGE
    assert f(4, 8, FAKE, 7, 0, spec(), FAKE, 8, None) == EINVAL   # ldx < F
    assert f(*ok, spec(), FAKE, 7, None) == EINVAL
    assert f(4, 8, None, 8, 0, spec(), FAKE, 8, None) == EINVAL
    assert f(4, 8, FAKE, 8, 0, spec(), FAKE, 9, None) == EINVAL   # in place, other stride
    assert f(0, 8, None, 8, 0, spec(), None, 8, None) == 0


def test_layernorm_affine_refusals(L):
    f = L.gcn_layernorm_affine_fwd
    assert f(4, 0, FAKE, 8, 0, None, None, 1e-5, None, FAKE, 8, None) == EINVAL
    assert f(4, 8, FAKE, 8, 7, None, None, 1e-5, None, FAKE, 8, None) == EINVAL
    assert f(4, 8, FAKE, 8, 0, None, None, -1e-5, None, FAKE, 8, None) == EINVAL
    assert f(4, 8, FAKE, 8, 0, None, None, float("nan"), None, FAKE, 8, None) == EINVAL
    assert f(4, 8, FAKE, 8, 0, None, None, 1e-5, spec(1.0), FAKE, 8, None) == EINVAL
    assert f(4, 8, FAKE, 4, 0, None, None, 1e-5, None, FAKE, 8, None) == EINVAL
    assert f(4, 8, FAKE, 8, 0, None, None, 1e-5, None, None, 8, None) == EINVAL
    assert f(4, 8, FAKE, 8, 0, None, None, 1e-5, None, FAKE, 16, None) == EINVAL
    assert f(1 << 31, 8, FAKE, 8, 0, None, None, 1e-5, None, FAKE, 8, None) == ERANGE
    assert f(0, 8, None, 8, 0, None, None, 1e-5, None, None, 8, None) == 0
    b = L.gcn_layernorm_affine_bwd
    other = ctypes.c_void_p(0x2000)
    assert b(4, 8, FAKE, 8, 0, None, 1e-5, None, other, 8, None, 0, None, None, None, None, None) == EINVAL
    assert b(4, 8, None, 8, 0, None, 1e-5, None, other, 8, FAKE, 8, None, None, None, None, None) == EINVAL
    assert b(4, 8, FAKE, 8, 0, None, 1e-5, None, None, 8, FAKE, 8, None, None, None, None, None) == EINVAL
    assert b(4, 8, FAKE, 8, 0, None, 1e-5, None, other, 4, FAKE, 8, None, None, None, None, None) == EINVAL
    assert b(4, 8, FAKE, 8, 0, None, 1e-5, None, other, 8, FAKE, 9, None, None, None, None, None) == EINVAL
    assert b(4, 8, FAKE, 8, 0, None, 1e-5, None, other, 8, other, 9, None, None, None, None, None) == EINVAL
    assert b(4, 8, FAKE, 8, 0, None, -1.0, None, other, 8, other, 8, None, None, None, None, None) == EINVAL
    # no rows and no sums wanted: nothing to do
    assert b(0, 8, None, 8, 0, None, 1e-5, None, None, 8, FAKE, 8, None, None, None, None, None) == 0


def test_gemm_grouped_refusals(L):
    def f(op=0, G=2, off=FAKE, rows=4, N=8, K=8, A=FAKE, lda=8, B=FAKE, ldb=8, dt=0, C=FAKE, ldc=8,
          dc=0, sw=64, work=None, size=None):
        return L.gcn_gemm_grouped(op, G, off, rows, N, K, A, lda, B, ldb, dt, C, ldc, dc, sw,
                                  work, size, None)
    for kw in (dict(op=3), dict(op=-1), dict(G=0), dict(G=65536), dict(rows=-1), dict(N=0),
               dict(K=0), dict(N=1 << 24), dict(K=1 << 24), dict(dt=2), dict(dc=2), dict(dc=1),
               dict(dt=1, dc=2), dict(op=2, dt=1, dc=1), dict(off=None), dict(A=None),
               dict(B=None), dict(C=None), dict(lda=7), dict(ldb=7), dict(ldc=7), dict(sw=-1),
               dict(op=1, ldb=7), dict(op=2, sw=63), dict(lda=1 << 41)):
        assert f(**kw) == EINVAL, kw
    assert f(rows=1 << 31) == ERANGE
    assert f(rows=0) == 0  # no rows: nothing to write
    assert f(work=FAKE) == EINVAL
    some = ctypes.c_int64(1 << 30)
    assert f(work=ctypes.c_void_p(0x1010), size=ctypes.byref(some)) == EINVAL  # 256-byte aligned
    assert L.gcn_layernorm_affine_bwd(4, 8, FAKE, 8, 0, None, 1e-5, None, ctypes.c_void_p(0x2000), 8, FAKE, 8,
                                      None, None, ctypes.c_void_p(0x1010), ctypes.byref(some), None) == EINVAL
    # what a call would use: nothing for rows times a matrix, the chunks' sums for a weight gradient
    size = ctypes.c_int64(-1)
    assert f(size=ctypes.byref(size)) == 0 and size.value == 0
    big = dict(op=2, rows=100000, N=256, K=256, lda=256, ldb=256, ldc=256, sw=65536)
    assert f(size=ctypes.byref(size), **big) == 0
    assert size.value % (256 * 256 * 4) == 0 and size.value > 0
    less = ctypes.c_int64(size.value - 256)
    assert f(work=FAKE, size=ctypes.byref(less), **big) == EINVAL


@pytest.mark.parametrize("rows,K,N,most", [
    (2449029, 512, 256, 350e6),     # 637 runs of two chunks
    (500000, 4096, 4096, 4.2e9),    # about 8192 rows to a run, 64 MB each
    (65536, 4096, 14336, 2.0e9), (131072, 16384, 16384, 18e9), (500000, 256, 256, 134e6)])
def test_grouped_weight_gradients_memory(L, rows, K, N, most):
    """The partial sums of fp32 weight gradients take about as much memory as those of the ungrouped product."""
    size = ctypes.c_int64(-1)
    assert L.gcn_gemm_grouped(2, 4, FAKE, rows, N, K, FAKE, K, FAKE, N, 0, FAKE, N, 0, K * N, None,
                              ctypes.byref(size), None) == 0
    assert 0 < size.value <= most


def test_grouped_more_tiles_than_a_launch(L):
    """Every kernel of the products refuses what one launch does not take before it starts."""
    def f(op, G, rows, N, K, dt, lda=None, ldb=None):
        ldb = ldb or (K if op == 1 else N)
        return L.gcn_gemm_grouped(op, G, FAKE, rows, N, K, FAKE, lda or K, FAKE, ldb, dt, FAKE, N, 0,
                                  K * N, None, None, None)
    top = (1 << 31) - 1
    for op in (0, 1):
        assert f(op, 2, top, 4, 4, 1) == ERANGE              # bf16, the general product
        assert f(op, 2, top, 4, 4, 0, lda=1 << 22) == ERANGE  # fp32 in rows far apart
        assert f(op, 1, 1 << 20, 1 << 23, 4, 1) == ERANGE    # many columns
        assert f(op, 2, top, 4096, 64, 1) == ERANGE and f(op, 2, top, 4096, 64, 0) == ERANGE
    assert f(2, 65535, 100, 1 << 23, 4, 1) == ERANGE




def test_grouped_narrow_weight_gradients_are_cut(L):
    """bf16 weight gradients of fewer than 8 columns have partial sums: several workgroups to a group."""
    for K, N in ((256, 4), (4, 256), (1, 1)):
        size = ctypes.c_int64(-1)
        assert L.gcn_gemm_grouped(2, 4, FAKE, 500000, N, K, FAKE, K, FAKE, N, 1, FAKE, N, 0, K * N, None,
                                  ctypes.byref(size), None) == 0
        assert size.value >= 100 * 4 * K * N


def test_row0_is_not_cut(L):
    """A row number that does not fit the call's is refused, not taken modulo 2^64."""
    import paper_2411_16025_amd as pkg
    for row0 in (1 << 64, (1 << 64) + 5, 1 << 63, -(1 << 63) - 1):
        with pytest.raises(ValueError):
            pkg.Dropout(0.5, 1, row0=row0)
    assert L.gcn_dropout(4, 8, FAKE, 8, 0, spec(row0=(1 << 63) - 1), FAKE, 8, None) == ERANGE


def test_grouped_weight_gradients_keep_their_workgroups(L):
    """A workgroup adds up several chunks only where 512 are left: of a small matrix every chunk but the
    first ones has a partial sum."""
    size = ctypes.c_int64(-1)
    rows, K, N = 176075, 47, 32
    assert L.gcn_gemm_grouped(2, 12, FAKE, rows, N, K, FAKE, K, FAKE, N, 0, FAKE, N, 0, K * N, None,
                              ctypes.byref(size), None) == 0
    assert size.value >= 480 * 4 * K * N
