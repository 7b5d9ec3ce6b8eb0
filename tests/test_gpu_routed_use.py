"""The routed layer's calls as programs use them: captured and replayed, on other streams, over more elements
than 32 bits count, again and again, with arguments that the binding refuses."""

import ctypes

import numpy as np
import pytest

import routed_ref as ref
from gpu_util import dev, host, note

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def G():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2411_16025_amd as pkg
    pkg.lib()
    return pkg


class Layer:
    """A training step of a routed layer: ids -> rows of a table -> router -> experts' products of rows kept in
    8 bits for the weights -> back, and all gradients. Without `products` the experts pass their rows on (H = F)
    and the logits are given: only the calls around gcn_gemm_grouped run."""

    def __init__(self, n, V, F, H, E, k, dtype, seed, products=True):
        import torch
        self.products = products
        r = np.random.default_rng(seed)
        self.n, self.V, self.E, self.k = n, V, E, k
        t = lambda *s: dev(r.standard_normal(s).astype(np.float32) / 8).to(dtype)  # noqa: E731
        self.table, self.Wr, self.W = t(V, F), t(1, F, E), t(E, F, H)
        self.ids = dev(ref.some_ids(r, n, V, "none"))
        self.mask = dev((r.random(n) < 0.9).astype(np.uint8))
        self.dy = t(n, H)
        self.dloss = torch.ones(1, device="cuda:0")
        self.whole = torch.tensor([0, n], device="cuda:0")
        self.z = t(n, E)

    def step(self, G):
        x = G.gcn_embed_fwd(self.table, self.ids, scale=4.0)
        z = G.gcn_gemm_grouped(G.GCN_GEMM_NN, self.whole, x, self.Wr) if self.products else self.z
        experts, w, counts, loss = G.gcn_route_fwd(z, self.k, mask=self.mask, coef=0.1, normalize=True)
        offsets, order, slot = G.gcn_group_ids(experts.view(-1), self.E)
        slot = slot.view(self.n, self.k)
        xs = G.gcn_embed_fwd(x, order, per=self.k)
        Q, S = G.gcn_pack8(xs)
        h = G.gcn_gemm_grouped(G.GCN_GEMM_NN, offsets, xs, self.W) if self.products else xs
        y = G.gcn_combine_fwd(h, slot, w)
        dh, dw = G.gcn_combine_bwd(h, slot, w, self.dy)
        dW = G.gcn_gemm_grouped_q8(offsets, Q, S, dh)
        dxs = G.gcn_gemm_grouped(G.GCN_GEMM_NT, offsets, dh, self.W) if self.products else dh
        dx = G.gcn_combine_fwd(dxs, slot)
        dz = G.gcn_route_bwd(z, experts, w, counts, dweights=dw, coef=0.1, normalize=True, dloss=self.dloss)
        dWr = dz
        if self.products:
            dx.add_(G.gcn_gemm_grouped(G.GCN_GEMM_NT, self.whole, dz, self.Wr))
            dWr = G.gcn_gemm_grouped(G.GCN_GEMM_TN, self.whole, x, dz)
        by_id, places, _ = G.gcn_group_ids(self.ids, self.V, slots=False)
        dT = G.gcn_embed_bwd(dx, by_id, places, scale=4.0)
        rest = G.gcn_unpack8(Q, S, out_dtype=x.dtype)
        # rows behind the last group are not defined: not compared
        return dict(x=x, experts=experts, w=w, counts=counts, loss=loss, offsets=offsets, order=order, slot=slot,
                    xs=xs, rest=rest, y=y, dw=dw, dW=dW, dx=dx, dz=dz, dWr=dWr, dT=dT)

    def change(self, seed):
        import torch
        r = np.random.default_rng(seed)
        self.ids.copy_(dev(ref.some_ids(r, self.n, self.V, ("skew", "none", "one")[seed % 3])))
        self.mask.copy_(dev((r.random(self.n) < (0.0 if seed == 2 else 0.8)).astype(np.uint8)))
        self.table.copy_(torch.randn(self.table.shape, device="cuda:0", dtype=torch.float32).to(self.table.dtype))
        self.dloss.fill_(1.0 + seed)


def same(got, want, what):
    import torch
    for k in want:
        a, b = got[k], want[k]
        assert torch.equal(a, b) or torch.equal(a.isnan(), b.isnan()) and torch.equal(
            a[~a.isnan()], b[~b.isnan()]), (what, k)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n,V,F,E,k", [(5000, 700, 96, 6, 2), (300, 5000, 64, 16, 4)])
def test_captured_layers(G, n, V, F, E, k, kind):
    """Two captured steps, replayed in turn with new inputs, eager work and synchronizations between the replays:
    every replay equals the eager step bit for bit. (bf16: without the products by group, whose captured bf16
    calls stay off while the cause of a fault of theirs is not known.)"""
    import torch
    note("captured routed layers n=%d %s" % (n, kind))
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    products = kind == "f32"
    H = F + 32 if products else F
    layers = [Layer(n, V, F, H, E, k, dtype, 1, products), Layer(n // 2 + 1, V, F, H, E, k, dtype, 2, products)]
    graphs, outs = [], []
    for la in layers:
        la.step(G)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            outs.append(la.step(G))
        graphs.append(g)
        torch.cuda.synchronize()
    for rep in range(4):
        for la, g, out in zip(layers, graphs, outs):
            la.change(rep)
            for v in out.values():
                v.zero_()
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            want = la.step(G)
            torch.cuda.synchronize()
            same(out, want, (rep, la.n))
    del graphs, outs


def test_captured_calls_need_work_memory(G):
    """A captured C call without work memory is refused where it needs some, and with the caller's runs."""
    import torch
    note("captured calls without work memory")
    n, V, F = 6000, 3000, 64
    ids = torch.randint(0, V, (n,), device="cuda:0", dtype=torch.int32)
    dy = torch.randn(n, F, device="cuda:0")
    off, order, _ = G.gcn_group_ids(ids, V)
    z = torch.randn(n, 16, device="cuda:0")
    ex, w, c, loss = G.gcn_route_fwd(z, 2, coef=1.0)
    Q, S = G.gcn_pack8(dy)
    whole = torch.tensor([0, n], device="cuda:0")
    dT, dW = torch.empty(V, F, device="cuda:0"), torch.empty(F, F, device="cuda:0")
    L = G.lib()
    calls = [
        lambda wk, sz, s: L.gcn_group_ids(n, ids.data_ptr(), V, off.data_ptr(), order.data_ptr(), None, wk, sz, s),
        lambda wk, sz, s: L.gcn_embed_bwd(n, F, V, off.data_ptr(), order.data_ptr(), dy.data_ptr(), F, 0, 1.0,
                                          dT.data_ptr(), F, 0, 0, wk, sz, s),
        lambda wk, sz, s: L.gcn_route_fwd(n, 16, z.data_ptr(), 16, 0, 2, 0, None, 1.0, ex.data_ptr(), w.data_ptr(),
                                          c.data_ptr(), loss.data_ptr(), wk, sz, s),
        lambda wk, sz, s: L.gcn_gemm_grouped_q8(1, whole.data_ptr(), n, F, F, Q.data_ptr(), F, S.data_ptr(), 2,
                                                dy.data_ptr(), F, 0, dW.data_ptr(), F, 0, wk, sz, s)]
    need = [ctypes.c_int64(-1) for _ in calls]
    for call, size in zip(calls, need):
        assert call(None, ctypes.byref(size), None) == 0 and size.value > 0
    work = [torch.empty(size.value, dtype=torch.uint8, device="cuda:0") for size in need]
    torch.cuda.synchronize()
    graph, st = torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        s = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
        for call, size, wk in zip(calls, need, work):
            st.append(call(None, None, s))
            st.append(call(wk.data_ptr(), ctypes.byref(size), s))
    assert st == [5, 0] * len(calls)
    want = [t.clone() for t in (off, order, ex, w, c, loss)] + [G.gcn_embed_bwd(dy, off, order),
                                                                G.gcn_gemm_grouped_q8(whole, Q, S, dy)[0]]
    for _ in range(3):
        for t in (off, order, ex, w, c, loss, dT, dW):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for t, v in zip((off, order, ex, w, c, loss, dT, dW), want):
            assert torch.equal(t, v)
    del graph


def test_other_streams_and_repeats(G):
    """A step on a stream of its own, with its inputs made there, equals that on the default stream; two at once
    on two streams do too; and repeated calls give the same bits."""
    import torch
    note("routed layer on other streams")
    la = Layer(4000, 600, 96, 100, 5, 2, torch.bfloat16, 3)
    lb = Layer(3000, 40, 64, 48, 8, 3, torch.float32, 4)
    wa, wb = la.step(G), lb.step(G)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(sa):
            a = la.step(G)
        with torch.cuda.stream(sb):
            b = lb.step(G)
        torch.cuda.synchronize()
        same(a, wa, "stream a")
        same(b, wb, "stream b")
    # the stream as an argument, and as a raw handle
    for s in (sa, sa.cuda_stream):
        off, order, slot = G.gcn_group_ids(la.ids, la.V, stream=s)
        x = G.gcn_embed_fwd(la.table, la.ids, scale=4.0, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(x, wa["x"])
        assert torch.equal(off[1:] - off[:-1], torch.bincount(la.ids[(la.ids >= 0) & (la.ids < la.V)].long(),
                                                              minlength=la.V))


def test_more_elements_than_32_bits_count(G):
    """Rows whose elements lie beyond 2^31 and 2^32 bytes and elements."""
    import torch
    note("large arrays")
    F, V = 1100, (1 << 32) // 1100 + 7   # a little over 2^32 elements
    T = torch.zeros((V, F), dtype=torch.bfloat16, device="cuda:0")
    ids = torch.tensor([V - 1, 0, V - 2, -1, V, V // 2, V - 1], dtype=torch.int32, device="cuda:0")
    rows = torch.randn(4, F, device="cuda:0").bfloat16()
    for i, v in enumerate((V - 1, 0, V - 2, V // 2)):
        T[v] = rows[i]
    Y = G.gcn_embed_fwd(T, ids, out_dtype=torch.float32)
    want = torch.stack([rows[0], rows[1], rows[2], rows[0] * 0, rows[0] * 0, rows[3], rows[0]]).float()
    assert torch.equal(Y, want)
    off, order, _ = G.gcn_group_ids(ids, V)
    T.fill_(3.0)
    G.gcn_embed_bwd(Y, off, order, dT=T)
    assert torch.equal(T[V - 1], (2 * rows[0].float()).bfloat16()) and torch.equal(T[V - 2], rows[2])
    assert torch.equal(T[0], rows[1]) and torch.equal(T[V // 2], rows[3])
    assert int((T != 0).any(1).sum()) == 4
    G.gcn_embed_bwd(Y, off, order, dT=T, accumulate=True)
    assert torch.equal(T[V - 2], 2 * rows[2]) and int((T != 0).any(1).sum()) == 4
    # back from places far behind
    slot = torch.tensor([[V - 1, V - 2], [0, -1], [V // 2, V]], dtype=torch.int32, device="cuda:0")
    w = torch.tensor([[1.0, 2.0], [3.0, 4.0], [0.5, 1.0]], device="cuda:0")
    y = G.gcn_combine_fwd(T, slot, w)
    t = T[torch.tensor([V - 1, V - 2, 0, V // 2], device="cuda:0")].float()
    assert torch.equal(y.float(), torch.stack([t[0] + 2 * t[1], 3 * t[2], 0.5 * t[3]]).bfloat16().float())
    dy = torch.randn(3, F, device="cuda:0").bfloat16()
    _, dw = G.gcn_combine_bwd(T, slot, w, dy, dZ=T)
    assert torch.equal(T[V - 2], (2 * dy[0].float()).bfloat16()) and float(dw[1, 1]) == 0.0
    # codes
    T[V // 2].copy_(rows[3])
    Q, S = G.gcn_pack8(T)
    some = torch.tensor([0, 1, V // 2, V - 2, V - 1], device="cuda:0")
    q, s = ref.pack8(host(T[some].float()))
    assert np.array_equal(host(Q[some]), q) and np.array_equal(host(S[some]), s)
    back = G.gcn_unpack8(Q, S, Y=T)
    assert np.array_equal(host(back[some].float()), ref.unpack8(q, s).astype(np.float32))
    B = torch.zeros((V, 8), dtype=torch.bfloat16, device="cuda:0")
    B[some] = torch.randn(5, 8, device="cuda:0").bfloat16()
    ends = torch.tensor([0, V - 2, V], device="cuda:0")
    C = host(G.gcn_gemm_grouped_q8(ends, Q, S, B)).astype(np.float64)
    x, b = ref.unpack8(q, s), host(B[some].float()).astype(np.float64)
    for g, r in enumerate((slice(0, 3), slice(3, 5))):
        want = x[r].T @ b[r]
        assert (np.abs(C[g] - want) <= 16 * ref.U * (np.abs(x[r]).T @ np.abs(b[r]))).all()


def test_long_batch_of_a_small_table(G):
    """Two million rows of forty-seven ids: the label table of a large graph."""
    import torch
    note("small table, long batch")
    n, V, F = 2449029, 47, 100
    ids = (torch.rand(n, device="cuda:0") ** 2 * V).int()
    dy = torch.randn(n, F, device="cuda:0")
    off, order, _ = G.gcn_group_ids(ids, V)
    dT = G.gcn_embed_bwd(dy, off, order, scale=0.5)
    want, mag = torch.zeros(V, F, dtype=torch.float64), torch.zeros(V, F, dtype=torch.float64)
    want.index_add_(0, ids.cpu().long(), dy.cpu().double())
    mag.index_add_(0, ids.cpu().long(), dy.cpu().double().abs())
    assert bool(((dT.cpu().double() - 0.5 * want).abs() <= 260 * ref.U * 0.5 * mag).all())
    # (chains of 256 at most: of random signs far closer)
    assert float((dT.cpu().double() - 0.5 * want).norm() / (0.5 * want).norm()) < 2e-6


def test_binding_refusals(G):
    import torch
    note("binding refusals")
    c = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda:0")  # noqa: E731
    i32, i64, u8, i8, b16 = torch.int32, torch.int64, torch.uint8, torch.int8, torch.bfloat16
    bad = [
        lambda: G.gcn_group_ids(c(4), 3), lambda: G.gcn_group_ids(c(4, 2, dt=i32), 3),
        lambda: G.gcn_group_ids(c(8, dt=i32)[::2], 3), lambda: G.gcn_group_ids(torch.zeros(4, dtype=i32), 3),
        lambda: G.gcn_group_ids(c(4, dt=i32), 0), lambda: G.gcn_group_ids(c(4, dt=i32), -1),
        lambda: G.gcn_embed_fwd(c(5, 8), c(4, dt=i64)), lambda: G.gcn_embed_fwd(c(5, 8, dt=i32), c(4, dt=i32)),
        lambda: G.gcn_embed_fwd(c(8, 5).t(), c(4, dt=i32)), lambda: G.gcn_embed_fwd(c(5, 8), c(4, dt=i32), per=0),
        lambda: G.gcn_embed_fwd(c(5, 8), c(4, dt=i32), Y=c(4, 7)),
        lambda: G.gcn_embed_fwd(c(5, 8), c(4, dt=i32), Y=c(4, 8), out_dtype=b16),
        lambda: G.gcn_embed_fwd(c(5, 8), c(4, dt=i32), scale=float("inf")),
        lambda: G.gcn_embed_fwd(c(5, 8), c(4, dt=i32), out_dtype=torch.float16),
        lambda: G.gcn_embed_bwd(c(4, 8), c(6, dt=i32), c(4, dt=i32)), lambda: G.gcn_embed_bwd(c(4, 8), c(6, dt=i64), c(3, dt=i32)),
        lambda: G.gcn_embed_bwd(c(4, 8), c(6, dt=i64), c(4, dt=i32), accumulate=True),
        lambda: G.gcn_embed_bwd(c(4, 8), c(6, dt=i64), c(4, dt=i32), dT=c(6, 8)),
        lambda: G.gcn_route_fwd(c(4, 8), 0), lambda: G.gcn_route_fwd(c(4, 8), 9), lambda: G.gcn_route_fwd(c(4, 1025), 1),
        lambda: G.gcn_route_fwd(c(4, 8), 2, mask=c(4)), lambda: G.gcn_route_fwd(c(4, 8), 2, mask=c(3, dt=u8)),
        lambda: G.gcn_route_bwd(c(4, 8), c(3, 2, dt=i32), c(4, 2)), lambda: G.gcn_route_bwd(c(4, 8), c(4, 2, dt=i32), c(4, 3)),
        lambda: G.gcn_route_bwd(c(4, 8), c(4, 2, dt=i32), c(4, 2), coef=1.0),
        lambda: G.gcn_route_bwd(c(4, 8), c(4, 2, dt=i32), c(4, 2), counts=c(8, dt=i64)),
        lambda: G.gcn_route_bwd(c(4, 8), c(4, 2, dt=i32), c(4, 2), dloss=c(2)),
        lambda: G.gcn_combine_fwd(c(6, 8), c(6, dt=i32)), lambda: G.gcn_combine_fwd(c(6, 8), c(3, 2, dt=i64)),
        lambda: G.gcn_combine_fwd(c(6, 8), c(3, 2, dt=i32), c(3, 3)), lambda: G.gcn_combine_fwd(c(6, 8), c(3, 2, dt=i32), c(3, 2, dt=b16)),
        lambda: G.gcn_combine_fwd(c(6, 8), c(3, 2, dt=i32), Y=c(3, 8, dt=b16)),
        lambda: G.gcn_combine_bwd(c(6, 8), c(3, 2, dt=i32), None, c(2, 8)),
        lambda: G.gcn_combine_bwd(c(6, 8), c(3, 2, dt=i32), None, c(3, 8), input_grad=False, weight_grad=False),
        lambda: G.gcn_pack8(c(4, 8, dt=i32)), lambda: G.gcn_pack8(c(8, 4).t()),
        lambda: G.gcn_unpack8(c(4, 40, dt=i8), c(4, 1, dt=u8)), lambda: G.gcn_unpack8(c(4, 40, dt=u8), c(4, 2, dt=u8)),
        lambda: G.gcn_unpack8(c(4, 40, dt=i8), c(4, 2, dt=u8), Y=c(4, 39)),
        lambda: G.gcn_gemm_grouped_q8(c(3, dt=i32), c(4, 40, dt=i8), c(4, 2, dt=u8), c(4, 8)),
        lambda: G.gcn_gemm_grouped_q8(c(3, dt=i64), c(4, 40, dt=i8), c(4, 1, dt=u8), c(4, 8)),
        lambda: G.gcn_gemm_grouped_q8(c(3, dt=i64), c(4, 40, dt=i8), c(4, 2, dt=u8), c(5, 8)),
        lambda: G.gcn_gemm_grouped_q8(c(3, dt=i64), c(4, 40, dt=i8), c(4, 2, dt=u8), c(4, 8), C=c(2, 40, 7)),
        lambda: G.gcn_gemm_grouped_q8(c(3, dt=i64), c(4, 40, dt=i8), c(4, 2, dt=u8), c(4, 8), C=c(2, 40, 8, dt=b16)),
    ]
    for i, f in enumerate(bad):
        with pytest.raises((TypeError, ValueError, G.GcnError)):
            f()
            pytest.fail("not refused: %d" % i)
    torch.cuda.synchronize()


def test_empty_and_single(G):
    """No rows at all, one row, one token that chose nothing."""
    import torch
    note("empty and single")
    e = lambda *s, dt=torch.float32: torch.empty(s, dtype=dt, device="cuda:0")  # noqa: E731
    off, order, slot = G.gcn_group_ids(e(0, dt=torch.int32), 4)
    assert host(off).tolist() == [0] * 5 and order.numel() == 0 and slot.numel() == 0
    T = torch.randn(5, 6, device="cuda:0")
    assert G.gcn_embed_fwd(T, e(0, dt=torch.int32)).shape == (0, 6)
    assert not bool(G.gcn_embed_bwd(e(0, 6), off, order).any())
    ex, w, c, loss = G.gcn_route_fwd(e(0, 4), 2, coef=1.0)
    assert ex.shape == (0, 2) and host(c).tolist() == [0] * 5 and float(loss) == 0.0
    assert G.gcn_combine_fwd(T, e(0, 2, dt=torch.int32)).shape == (0, 6)
    assert not bool(G.gcn_combine_fwd(e(0, 6), torch.zeros((3, 2), dtype=torch.int32, device="cuda:0")).any())
    Q, S = G.gcn_pack8(e(0, 40))
    assert Q.shape == (0, 40) and S.shape == (0, 2) and G.gcn_unpack8(Q, S).shape == (0, 40)
    assert not bool(G.gcn_gemm_grouped_q8(torch.zeros(3, dtype=torch.int64, device="cuda:0"), Q, S, e(0, 9)).any())
    off, order, slot = G.gcn_group_ids(torch.tensor([-1], dtype=torch.int32, device="cuda:0"), 2)
    assert host(off).tolist() == [0, 0, 0] and host(order).tolist() == [-1] and host(slot).tolist() == [-1]
    assert not bool(G.gcn_embed_fwd(T, order).any())
    torch.cuda.synchronize()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_route_gradient_in_place_and_in_parts(G, kind):
    """The logits' gradient in the logits' place; that of the weights alone and that of the loss alone, whose
    sum it is."""
    import torch
    note("router gradient in place")
    n, E, k = 513, 20, 3
    r = np.random.default_rng(2)
    z = dev(r.standard_normal((n, E)).astype(np.float32)).to(torch.float32 if kind == "f32" else torch.bfloat16)
    dw = dev(r.standard_normal((n, k)).astype(np.float32))
    for normalize in (False, True):
        ex, w, c, _ = G.gcn_route_fwd(z, k, coef=0.5, normalize=normalize)
        both = G.gcn_route_bwd(z, ex, w, c, dweights=dw, coef=0.5, normalize=normalize)
        one = G.gcn_route_bwd(z, ex, w, dweights=dw, normalize=normalize).double()
        two = G.gcn_route_bwd(z, ex, w, c, coef=0.5, normalize=normalize).double()
        # three roundings to the type, and those of fp32 sums of some terms of this size
        unit = (one.abs() + two.abs()) * (ref.HALF[kind] if kind == "bf16" else 0) * 2 + 200 * ref.U
        assert bool(((one + two - both.double()).abs() <= unit).all())
        assert not bool(G.gcn_route_bwd(z, ex, w, normalize=normalize).any())
        y = z.clone()
        assert G.gcn_route_bwd(y, ex, w, c, dweights=dw, coef=0.5, normalize=normalize, dlogits=y) is y
        assert torch.equal(y, both)


def test_only_what_is_asked_for(G):
    """Outputs that are left out, and given ones: rows of a wider matrix, whose other columns stay."""
    import torch
    note("outputs left out")
    n, k, F, rows = 50, 2, 40, 100
    r = np.random.default_rng(4)
    Z, dY = dev(r.standard_normal((rows, F)).astype(np.float32)), dev(r.standard_normal((n, F)).astype(np.float32))
    slot = dev(r.permutation(rows)[:n * k].reshape(n, k).astype(np.int32))
    w = dev(r.random((n, k)).astype(np.float32))
    dZ, dw = G.gcn_combine_bwd(Z, slot, w, dY)
    a, none = G.gcn_combine_bwd(Z, slot, w, dY, weight_grad=False)
    assert none is None and torch.equal(a, dZ)
    none, b = G.gcn_combine_bwd(Z, slot, w, dY, input_grad=False)
    assert none is None and torch.equal(b, dw)
    assert torch.equal(G.gcn_combine_fwd(Z, slot), G.gcn_combine_fwd(Z, slot, torch.ones_like(w)))
    wide = torch.full((n, F + 7), 3.0, device="cuda:0")
    G.gcn_combine_fwd(Z, slot, w, Y=wide[:, 3:3 + F])
    assert torch.equal(wide[:, 3:3 + F], G.gcn_combine_fwd(Z, slot, w))
    assert bool((wide[:, :3] == 3).all()) and bool((wide[:, 3 + F:] == 3).all())
    ids = dev(r.integers(0, 9, n).astype(np.int32))
    off, order, slots = G.gcn_group_ids(ids, 9, slots=False)
    assert slots is None
    dT = torch.ones((9, F), device="cuda:0").bfloat16()
    G.gcn_embed_bwd(dY, off, order, dT=dT, accumulate=True)
    want = 1 + G.gcn_embed_bwd(dY, off, order).double()
    # the sum rounded to fp32, and with the one to bf16: half a step of each
    assert bool(((dT.double() - want).abs() <= want.abs() * 1.01 * 2.0 ** -8 + 1e-5).all())
    ex, w2, c, loss = G.gcn_route_fwd(Z, 3)
    assert loss is None and torch.equal(ex, G.gcn_route_fwd(Z, 3, coef=1.0)[0])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_neighbouring_columns(G, dtype):
    """Outputs that lie in other columns of their inputs' rows, and at their end."""
    import torch
    note("neighbouring columns %s" % dtype)
    n, F, k = 60, 40, 2
    r = np.random.default_rng(6)
    dt = getattr(torch, dtype)
    both = dev(r.standard_normal((2 * n, 2 * F + 8)).astype(np.float32)).to(dt)
    ids = dev(r.permutation(n).astype(np.int32))
    left, right, below = both[:n, :F], both[:n, F:2 * F], both[n:, :F]
    want = G.gcn_embed_fwd(left.clone(), ids, scale=0.5)
    for Y in (right, below, both[n - 1:2 * n - 1, F:2 * F]):
        keep = left.clone()
        assert torch.equal(G.gcn_embed_fwd(left, ids, scale=0.5, Y=Y), want) and torch.equal(left, keep)
    off, order, slot = G.gcn_group_ids(ids, n)
    assert torch.equal(G.gcn_embed_bwd(left, off, order, dT=right), G.gcn_embed_bwd(left.clone(), off, order, out_dtype=dt))
    slot = slot[:n // k * k].view(-1, k)
    w = dev(r.random(slot.shape).astype(np.float32))
    want = G.gcn_combine_fwd(left.clone(), slot, w)
    assert torch.equal(G.gcn_combine_fwd(left, slot, w, Y=right[:n // k]), want)
    dY = right[:n // k].clone()
    dZ, dw = G.gcn_combine_bwd(left, slot, w, dY, dZ=torch.zeros_like(left))
    right.zero_()
    got, dw2 = G.gcn_combine_bwd(left, slot, w, dY, dZ=right)
    assert torch.equal(got, dZ) and torch.equal(dw2, dw)
    # the weights' gradients in the weights' place
    st = G.lib().gcn_combine_bwd(n // k, k, F, left.data_ptr(), n, left.stride(0), 0 if dtype == "float32" else 1, slot.data_ptr(),
                                 w.data_ptr(), dY.data_ptr(), F, right.data_ptr(), right.stride(0), w.data_ptr(), None)
    torch.cuda.synchronize()
    assert st == 0 and torch.equal(w, dw) and torch.equal(right, dZ)
    z = both[:n, :F]
    ex, wt, c, _ = G.gcn_route_fwd(z, k, coef=1.0)
    want = G.gcn_route_bwd(z.clone(), ex, wt, c, coef=1.0)
    assert torch.equal(G.gcn_route_bwd(z, ex, wt, c, coef=1.0, dlogits=right), want)
    Q, S = G.gcn_pack8(left)
    assert torch.equal(G.gcn_unpack8(Q, S, Y=right), G.gcn_unpack8(Q, S, out_dtype=dt))
    for f in (lambda: G.gcn_embed_fwd(left, ids, Y=both[1:n + 1, :F]), lambda: G.gcn_embed_fwd(left, ids, Y=both[:n, 1:F + 1]),
              lambda: G.gcn_embed_bwd(left, off, order, dT=both[:n, F - 1:2 * F - 1]),
              lambda: G.gcn_combine_fwd(left, slot, w, Y=both[n - 1:n - 1 + n // k, :F]),
              lambda: G.gcn_combine_bwd(left, slot, w, dY, dZ=both[1:n + 1, :F]),
              lambda: G.gcn_route_bwd(z, ex, wt, c, coef=1.0, dlogits=both[1:n + 1, :F])):
        with pytest.raises(G.GcnError):
            f()
    torch.cuda.synchronize()
