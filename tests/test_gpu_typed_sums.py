"""Sums of the typed layer's operators where a lost term, a bias or an idle lane would show:
against 64 bits, and whole numbers exactly."""

import numpy as np
import pytest

import typed_ref as ref
from gpu_util import dev, host, note
from test_gpu_typed import KINDS, back, rows, tdtype, values, weights, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2411_16025_amd as pkg
    pkg.lib()
    return pkg


# ---- LayerNorm without eps -------------------------------------------------------------

# rows that do not fill the last workgroup's slots, widths that fill their lanes and do not
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,F", [(5, 64), (3, 7), (17, 100), (33, 128), (301, 256), (7, 300), (9, 1024),
                                 (6, 1000), (3, 2048), (2, 9000), (2, 16400)])
def test_layernorm_without_eps(G, n, F, kind):
    """eps = 0, and one whose root lies beyond fp32: rows with a deviation have all their values, and no
    row that is not there takes part in the weights' sums."""
    x, dy = values(n + F, n, F, kind, 1.5, 0.5), values(n + F + 1, n, F, kind)
    gamma, beta = weights(F, F)
    for eps, p in ((0.0, 0.0), (1e-100, 0.25)):
        note("norm without eps n=%d F=%d %s eps=%g" % (n, F, kind, eps))
        drop = G.Dropout(p, 3, 1) if p else None
        f = ref.factor(n, F, p, 3, 1) if p else 1.0
        X, dY = rows(x, kind), rows(dy, kind)
        Y = G.gcn_layernorm_affine_fwd(X, dev(gamma), dev(beta), eps, drop)
        within(back(Y), ref.norm_fwd(x, gamma, beta, eps, f),
               ref.norm_fwd_bound(x, gamma, beta, eps, f, kind), "Y")
        dx, dg, db = ref.norm_bwd(x, dy, gamma, eps, f)
        bx, bg, bb = ref.norm_bwd_bound(x, dy, gamma, eps, f, kind)
        dX, dgamma, dbeta = G.gcn_layernorm_affine_bwd(X, dY, dev(gamma), eps, drop)
        within(back(dX), dx, bx, "dX")
        within(back(dgamma), dg, bg, "dgamma")
        within(back(dbeta), db, bb, "dbeta")


# ---- weight gradients of many rows -------------------------------------------------------


def product64(x, dy, step=100000):
    """x^T dy in 64 bits, by pieces of the rows, on the GPU."""
    import torch
    c = torch.zeros(x.shape[1], dy.shape[1], dtype=torch.float64, device="cuda:0")
    for i in range(0, x.shape[0], step):
        c += x[i:i + step].double().t().contiguous() @ dy[i:i + step].double()
    return c


@pytest.mark.parametrize("n,K,N", [(2449029, 256, 96), (1000000, 256, 96), (500000, 300, 300),
                                   (500000, 512, 256), (300000, 70, 65)])
def test_weight_gradients_as_close_as_one_product(G, n, K, N):
    """gcn_gemm_f32's sums: a group's weight gradient is as close to 64 bits (in the matrices' norm) as
    that product of all rows; 5% for another order of the partial sums. Of a part of the rows too, against the
    product of all: in chunks of r rows each element of a chunk's sum has an error e(r) of its own
    sign, so that m chunks have e(r) sqrt(m) and the result, of independent terms, grows as sqrt(m) as
    well: the ratio is the chunk's, whatever m is."""
    import torch
    note("dW precision n=%d %dx%d" % (n, K, N))
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(n + K)
    x = torch.randn(n, K, generator=gen, device="cuda:0")
    dy = torch.randn(n, N, generator=gen, device="cuda:0")
    cut = n // 3 + 7
    ends = torch.tensor([0, n, n], device="cuda:0"), torch.tensor([0, cut, n], device="cuda:0")
    err = lambda c, want: float((c.double() - want).norm() / want.norm())  # noqa: E731
    want = product64(x, dy)
    most = err(G.gcn_gemm_f32(G.GCN_GEMM_TN, x, dy), want)
    one = G.gcn_gemm_grouped(G.GCN_GEMM_TN, ends[0], x, dy)
    note("dW error %.3e, one product %.3e" % (err(one[0], want), most))
    assert err(one[0], want) <= 1.05 * most and not one[1].any()
    two = G.gcn_gemm_grouped(G.GCN_GEMM_TN, ends[1], x, dy)
    for c, rows_ in ((two[0], slice(0, cut)), (two[1], slice(cut, n))):
        want = product64(x[rows_], dy[rows_])
        note("dW error of a part %.3e" % err(c, want))
        assert err(c, want) <= 1.05 * most


def whole(gen, kind, *shape):
    """Whole numbers from -3 to 3: sums of their products below 2^24 are exact in any order."""
    import torch
    return torch.randint(-3, 4, shape, generator=gen, device="cuda:0").to(tdtype(kind))


def cuts(sizes):
    return np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)


# several chunks of a group: a workgroup for each, and runs of them, by tiles shared among the XCDs and not
@pytest.mark.parametrize("kind,sizes,K,N", [
    ("f32", [140000, 5], 136, 132), ("f32", [9000, 2500, 0], 40, 70), ("f32", [120000], 256, 96),
    ("f32", [30011, 0, 5, 31984], 2047, 2050), ("f32", [70001, 129999], 1024, 1024),
    ("f32", [100003, 0, 100000], 8192, 64), ("f32", [150000, 50010], 8200, 32),
    ("bf16", [140000, 5], 136, 132), ("bf16", [9000, 2500, 0], 40, 70), ("bf16", [70001, 9], 520, 264),
    ("bf16", [70001, 0, 30000], 515, 517), ("bf16", [200003], 64, 64),
    ("bf16", [0, 70001, 0, 1, 30000], 256, 4), ("bf16", [150000, 7], 7, 130), ("bf16", [99999, 31], 1, 1),
    ("bf16", [1000, 0, 2000] * 30, 70, 3)])
def test_weight_gradients_exact(G, kind, sizes, K, N):
    """No row, chunk or operand part is lost, doubled or misplaced."""
    import torch
    note("dW exact %s sizes=%s K=%d N=%d" % (kind, sizes, K, N))
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(K)
    n, ends = sum(sizes), cuts(sizes)
    x, dy = whole(gen, kind, n, K), whole(gen, kind, n, N)
    got = G.gcn_gemm_grouped(G.GCN_GEMM_TN, dev(ends), x, dy)
    for g in range(len(sizes)):
        r = slice(int(ends[g]), int(ends[g + 1]))
        assert torch.equal(got[g].double(), product64(x[r], dy[r])), g


# ---- roundings as they add up -----------------------------------------------------------------


@pytest.mark.parametrize("op,kind,sizes,K,N,longest", [
    (0, "f32", [9000, 0, 500], 516, 200, 516), (1, "f32", [9000, 0, 500], 4096, 130, 4096),
    (0, "f32", [33000, 2000], 100, 256, 100), (0, "f32", [3] * 40, 700, 300, 700),
    (2, "f32", [140000, 5], 136, 132, 2048), (2, "f32", [70001, 129999], 1024, 1024, 4096),
    (2, "f32", [9000, 2500, 0], 40, 70, 2048),
    (0, "bf16", [9000, 0, 500], 1032, 520, 1032), (1, "bf16", [9000, 0, 500], 4099, 261, 4099),
    (0, "bf16", [3] * 40, 700, 300, 700), (2, "bf16", [140000, 5], 136, 132, 65536),
    (2, "bf16", [70001, 9], 520, 264, 65536), (2, "bf16", [150000, 7], 7, 130, 4096)])
def test_products_of_normal_values(G, op, kind, sizes, K, N, longest):
    """Errors as independent roundings make them, in the matrix's norm. A chain of m normal products, r
    roundings to every 16 of them, has partial sums of sqrt(16 k) after 16 k, so an error of
    U / sqrt(3) sqrt(r sum 16 k) = U sqrt(r / 96) m against sqrt(m): U sqrt(r m / 96). r is 6 of the three parts
    (the products left out of them are below a rounding), 4 of the fp32 instruction, 16 of multiplications
    one by one: twice 0.41 sqrt(m) covers all, and a row, a chunk or a part less is thousands of times that."""
    import torch
    note("normal values op=%d %s sizes=%s K=%d N=%d" % (op, kind, sizes[:4], K, N))
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(K * 7 + N)
    n, ends, t = sum(sizes), cuts(sizes), tdtype(kind)
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda:0").to(t)  # noqa: E731
    a = normal(n, K)
    b = normal(n, N) if op == 2 else normal(len(sizes), K, N) if op == 0 else normal(len(sizes), N, K)
    got = G.gcn_gemm_grouped(op, dev(ends), a, b, out_dtype=torch.float32)
    worst = ref.U * (1 + 0.82 * np.sqrt(longest))
    for g in range(len(sizes)):
        r = slice(int(ends[g]), int(ends[g + 1]))
        if op == 2:
            c, want = got[g], product64(a[r], b[r])
        else:
            w = b[g].double() if op == 0 else b[g].double().t().contiguous()
            c, want = got[r], a[r].double() @ w
        if want.numel() and sizes[g]:
            err = float((c.double() - want).norm() / want.norm())
            if sizes[g] > 100:
                note("error %.2e, at most %.2e" % (err, worst))
            assert err <= worst, (g, err)
        elif op == 2:
            assert not c.any()


# ---- long inner sizes ----------------------------------------------------------------------


@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("n,K,N,positive", [(8300, 5000, 160, False), (8300, 20000, 160, True),
                                            (8300, 20003, 130, False), (8300, 300007, 160, True),
                                            (7000, 1200003, 160, True)])
def test_long_inner_sizes(G, op, n, K, N, positive):
    """fp32 products by group are as close to 64 bits as gcn_gemm_f32's, which takes the fp32
    instruction there; also of positive operands, whose sums keep every bias (5% for another order)."""
    import torch
    note("long inner size op=%d K=%d positive=%d" % (op, K, positive))
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(K)
    a = torch.randn(n, K, generator=gen, device="cuda:0")
    b = torch.randn(2, K, N, generator=gen, device="cuda:0")
    if positive:
        a.abs_().add_(0.5)
        b.abs_().add_(0.5)
    ends = torch.tensor([0, n - 3000, n], device="cuda:0")
    w = b if op == 0 else b.transpose(1, 2).contiguous()
    got = G.gcn_gemm_grouped(op, ends, a, w)
    for g, r in enumerate((slice(0, n - 3000), slice(n - 3000, n))):
        want = torch.zeros(r.stop - r.start, N, dtype=torch.float64, device="cuda:0")
        for k in range(0, K, 20000):
            want += a[r, k:k + 20000].double() @ b[g, k:k + 20000].double()
        err = lambda c: float((c.double() - want).norm() / want.norm())  # noqa: E731
        one = err(G.gcn_gemm_f32(op, a[r].contiguous(), w[g]))
        note("error %.3e, one product %.3e" % (err(got[r]), one))
        assert err(got[r]) <= 1.05 * one


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("op", [0, 1])
@pytest.mark.parametrize("n,K,N", [(8300, 4096, 160), (8300, 16384, 130), (8300, 16385, 160),
                                   (40000, 32801, 256), (8300, 49153, 33), (9000, 20007, 300)])
def test_long_inner_sizes_exact(G, op, kind, n, K, N):
    """Whole numbers: nothing of the inner size is lost or taken twice, rows of no group are left."""
    import torch
    note("long inner size exact op=%d K=%d N=%d %s" % (op, K, N, kind))
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(K + N)
    a, b = whole(gen, kind, n, K), whole(gen, kind, 2, K, N)
    ends = [3, n // 2, n - 2]
    w = b if op == 0 else b.transpose(1, 2).contiguous()
    got = torch.full((n, N), 7.0, device="cuda:0")
    G.gcn_gemm_grouped(op, dev(np.array(ends, np.int64)), a, w, got, out_dtype=torch.float32)
    assert bool((got[:3] == 7.0).all()) and bool((got[n - 2:] == 7.0).all())
    for g in range(2):
        r = slice(ends[g], ends[g + 1])
        want = torch.zeros(r.stop - r.start, N, dtype=torch.float64, device="cuda:0")
        for k in range(0, K, 20000):
            want += a[r, k:k + 20000].double() @ b[g, k:k + 20000].double()
        assert torch.equal(got[r].double(), want), g


def test_long_inner_size_special_values(G):
    """Infinities and NaN of one piece of the inner size reach their own sums and no others."""
    import torch
    note("long inner size special values")
    n, K, N = 8300, 33000, 140
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(1)
    a, b = whole(gen, "f32", n, K), whole(gen, "f32", 1, K, N).abs() + 1
    a[5, 20000], a[700, 3], a[700, 32999], a[8000, 16384] = np.inf, np.inf, -np.inf, np.nan
    got = G.gcn_gemm_grouped(0, dev(np.array([0, n], np.int64)), a, b)
    assert bool(torch.isposinf(got[5]).all())
    assert bool(torch.isnan(got[700]).all()) and bool(torch.isnan(got[8000]).all())
    rest = torch.ones(n, dtype=torch.bool, device="cuda:0")
    rest[[5, 700, 8000]] = False
    assert torch.equal(got[rest].double(), a[rest].double() @ b[0].double())


# ---- sizes of the general product ------------------------------------------------------------


@pytest.mark.parametrize("op", [0, 1, 2])
def test_more_columns_than_a_second_axis(G, op):
    """More than 65,535 tiles of 64 columns (NN, TN) or rows of C (TN): bf16 rows of 2^22 elements and more
    take the general product."""
    import torch
    wide = (1 << 22) + 70
    note("general product, many tiles op=%d" % op)
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(op)
    if op == 2:  # both ways round
        for K, N in ((wide, 3), (3, wide)):
            x, dy = whole(gen, "bf16", 70, K), whole(gen, "bf16", 70, N)
            got = G.gcn_gemm_grouped(2, dev(np.array([0, 30, 69], np.int64)), x, dy)
            for g, r in enumerate((slice(0, 30), slice(30, 69))):
                assert torch.equal(got[g], x[r].float().t().contiguous() @ dy[r].float())
        return
    n, K = 130, 9
    a = whole(gen, "bf16", n, K)
    b = whole(gen, "bf16", 1, K, wide) if op == 0 else whole(gen, "bf16", 1, wide, K)
    got = G.gcn_gemm_grouped(op, dev(np.array([0, n], np.int64)), a, b, out_dtype=torch.float32)
    w = b[0].float() if op == 0 else b[0].float().t()
    for c in range(0, wide, 1 << 20):  # (by pieces: the library's product of 2 GB leaves a part of it zero)
        assert torch.equal(got[:, c:c + (1 << 20)], a.float() @ w[:, c:c + (1 << 20)].contiguous()), c


# ---- memory ----------------------------------------------------------------------------------


@pytest.mark.parametrize("kind", KINDS)
def test_captured_calls_record_kernels_only(G, kind):
    """A captured gradient takes its work memory from the graph's own: no memory is allocated, freed, set
    or copied by its nodes. (The graph is looked at and not launched.)"""
    import ctypes
    import torch
    note("captured nodes %s" % kind)
    hip = ctypes.CDLL("libamdhip64.so")
    t, n, K, N = tdtype(kind), 9000, 72, 136
    x, dy = dev(values(1, n, K, kind)).to(t), dev(values(2, n, N, kind)).to(t)
    w = dev(np.ones((2, K, N), np.float32)).to(t)
    ends = dev(np.array([0, 4000, n], np.int64))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        out = [G.gcn_gemm_grouped(G.GCN_GEMM_NT, ends, dy, w), G.gcn_gemm_grouped(G.GCN_GEMM_TN, ends, x, dy),
               *G.gcn_layernorm_affine_bwd(x, x, None, 1e-5, G.Dropout(0.5, 1))]
    raw, count = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t(0)
    assert hip.hipGraphGetNodes(raw, None, ctypes.byref(count)) == 0 and count.value >= 5
    nodes = (ctypes.c_void_p * count.value)()
    assert hip.hipGraphGetNodes(raw, nodes, ctypes.byref(count)) == 0
    for node in nodes:
        kind_of = ctypes.c_int(-1)
        assert hip.hipGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind_of)) == 0
        assert kind_of.value == 0  # hipGraphNodeTypeKernel
    del graph, out


@pytest.mark.parametrize("op,n,K,N", [(0, 2400, 2049, 4001), (1, 2400, 2049, 4001), (2, 70001, 515, 517),
                                      (2, 2400, 2049, 4001), (2, 40000, 1025, 700)])
def test_same_bits_without_copies(G, op, n, K, N):
    """Large bf16 products of odd widths, with work memory for the aligned copies and with too little for
    them: the same bits."""
    import ctypes
    import torch
    note("same bits without copies op=%d %d %d %d" % (op, n, K, N))
    t, L = torch.bfloat16, G.lib()
    ends = dev(np.array([0, n * 7 // 12, n * 7 // 12, n], np.int64))
    A = dev(values(50, n, K, "bf16")).to(t)
    if op == 2:
        B, C = dev(values(60, n, N, "bf16")).to(t), (3, K, N)
    else:
        w = np.random.default_rng(7).standard_normal((3, K, N) if op == 0 else (3, N, K))
        B, C = dev(w.astype(np.float32)).to(t), (n, N)
    pieces = sum(r * ((c + 7) // 8) for r, c in ((n, K), B.reshape(-1, B.shape[-1]).shape) if c % 8)

    def call(out, work, size):
        return L.gcn_gemm_grouped(op, 3, ends.data_ptr(), n, N, K, A.data_ptr(), K, B.data_ptr(),
                                  B.shape[-1], 1, out.data_ptr(), N, 0, K * N, work, ctypes.byref(size),
                                  torch.cuda.current_stream().cuda_stream)
    need = ctypes.c_int64(-1)
    got = [torch.full(C, 7.0, device="cuda:0") for _ in range(2)]
    assert call(got[0], None, need) == 0
    less = ctypes.c_int64(need.value - (16 * pieces + 255) // 256 * 256)
    assert pieces > 0 and 0 <= less.value < 16 * pieces
    work = torch.empty(need.value, dtype=torch.uint8, device="cuda:0")
    assert call(got[0], work.data_ptr(), need) == 0
    assert call(got[1], work.data_ptr(), less) == 0
    assert torch.equal(*got)


# ---- the caller's stream ---------------------------------------------------------------------


def test_current_stream_by_either_name(G, monkeypatch):
    """Calls run on the current stream, whether or not torch has the quicker name for its handle."""
    import torch
    from paper_2411_16025_amd import gcnagg
    note("current stream")
    side = torch.cuda.Stream()
    for raw in (gcnagg._raw_stream, None):
        monkeypatch.setattr(gcnagg, "_raw_stream", raw)
        for s in (torch.cuda.default_stream(), side):
            with torch.cuda.stream(s):
                got = gcnagg._stream(None)
                assert (getattr(got, "value", got) or 0) == s.cuda_stream
