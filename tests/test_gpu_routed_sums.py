"""Sums of the routed layer's operators as close to 64 bits as their roundings make them, where a bound of the
worst case would hide a lost row, a longer chain or a bias."""

import numpy as np
import pytest

import routed_ref as ref
from gpu_util import dev, host, note

pytestmark = pytest.mark.gpu

U = ref.U


@pytest.fixture(scope="module")
def G():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    import paper_2411_16025_amd as pkg
    pkg.lib()
    return pkg


def drawn(seed):
    import torch
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    return gen


def product64(x, dy, step=50000):
    """x^T dy in 64 bits, by pieces of the rows, on the GPU."""
    import torch
    c = torch.zeros(x.shape[1], dy.shape[1], dtype=torch.float64, device="cuda:0")
    for i in range(0, x.shape[0], step):
        c += x[i:i + step].double().t().contiguous() @ dy[i:i + step].double()
    return c


def off(got, want):
    """The error in the matrix's norm."""
    return float((got.double() - want).norm() / want.norm())


# ---- products from rows in 8 bits ---------------------------------------------------------

# kind, groups' rows, K, N, rows of the chunks that the sizes lead to
PRODUCTS = [("f32", [140000, 5], 136, 132, 1216), ("f32", [70001, 129999], 1024, 1024, 4608), ("f32", [1000000], 100, 256, 4096),
            ("f32", [9000, 2500, 0], 40, 70, 256), ("f32", [500000], 64, 64, 1088), ("f32", [150000, 7], 7, 130, 448),
            ("f32", [300000, 1], 2048, 1024, 7936), ("f32", [3500] * 40, 512, 512, 4096),
            ("bf16", [140000, 5], 136, 131, 1216), ("bf16", [70001, 9], 520, 264, 1792), ("bf16", [1000000], 100, 256, 4096),
            ("bf16", [150000, 7], 7, 130, 448), ("bf16", [300000, 1], 2048, 1024, 7936), ("bf16", [3500] * 40, 512, 512, 2368)]


@pytest.mark.parametrize("sign", ["normal", "positive"])
@pytest.mark.parametrize("kind,sizes,K,N,longest", PRODUCTS)
def test_products_from_8_bits(G, kind, sizes, K, N, longest, sign):
    """Independent roundings, of which a chain of m products has r to every 16: at most 16, one by one, and 3 of the
    three parts. Of normal values the sum of 16 k products is sqrt(16 k), so the chain's error is U / sqrt(3)
    sqrt(r sum 16 k) = U sqrt(r / 96) m against sqrt(m): at most 0.41 sqrt(m) U. Of positive ones it grows
    as k: U sqrt(r m / 144) of the sum, at most 0.34 sqrt(m) U; and the matrix core's rounding down, at most
    2^-8 of the last bit (2 U) of half the sum on average, r m / 16 times: r m 2^-12 U, 3 m 2^-12 U, which the
    chunks' signs may leave whole in a group of one. Twice the random part, and 3 U of the chunks' join and the
    result. A chunk of 100 rows less or twice would be thousands of U."""
    import torch
    note("8-bit products %s %s K=%d N=%d %s" % (kind, sizes[:4], K, N, sign))
    gen, n = drawn(K * 7 + N), sum(sizes)
    dt = torch.float32 if kind == "f32" else torch.bfloat16

    def some(F):
        v = torch.randn(n, F, generator=gen, device="cuda:0")
        return (v if sign == "normal" else v.abs()).to(dt)
    Q, S = G.gcn_pack8(some(K))
    x, dy = G.gcn_unpack8(Q, S), some(N)
    ends = np.concatenate([[0], np.cumsum(sizes)])
    got = G.gcn_gemm_grouped_q8(dev(ends), Q, S, dy)
    for g, rows in enumerate(sizes):
        if rows == 0:
            assert not bool(got[g].any())
            continue
        m = min(rows, longest)
        bound = 3 + 0.82 * m ** 0.5 if sign == "normal" else 3 + 0.68 * m ** 0.5 + 3 * m * 2.0 ** -12
        r = slice(int(ends[g]), int(ends[g + 1]))
        err = off(got[g], product64(x[r], dy[r]))
        note("group %d: %.1f U of %.1f" % (g, err / U, bound))
        assert err <= bound * U, (g, err / U, bound)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_longest_chunks(G, kind):
    """400,000 rows, 8192 x 8192: chunks of 65,536 rows, the longest there are; a part of the result."""
    import torch
    note("8-bit products, longest chunks %s" % kind)
    gen, n, F, m = drawn(5), 400000, 8192, 65536
    dt = torch.float32 if kind == "f32" else torch.bfloat16
    Q = torch.randint(-127, 128, (n, F), generator=gen, device="cuda:0", dtype=torch.int8)
    S = torch.randint(119, 122, (n, F // 32), generator=gen, device="cuda:0", dtype=torch.uint8)
    dy = torch.empty(n, F, device="cuda:0", dtype=dt)
    for i in range(0, n, 50000):
        dy[i:i + 50000] = torch.randn(50000, F, generator=gen, device="cuda:0")
    got = G.gcn_gemm_grouped_q8(torch.tensor([0, n], device="cuda:0"), Q, S, dy)[0]
    for k, c in ((0, 0), (8128, 4096), (1000, 8128)):
        unit = (S[:, k // 32:(k + 95) // 32].double() - 127).exp2().repeat_interleave(32, 1)
        x = Q[:, k // 32 * 32:k // 32 * 32 + unit.shape[1]].double() * unit
        x = x[:, k % 32:k % 32 + 64]
        want = product64(x, dy[:, c:c + 64])
        err = off(got[k:k + x.shape[1], c:c + 64], want)
        note("%.1f U" % (err / U))
        assert err <= (3 + 0.82 * m ** 0.5) * U


# ---- the table's gradient -------------------------------------------------------------------


@pytest.mark.parametrize("kd", ["f32", "bf16"])
@pytest.mark.parametrize("kt", ["f32", "bf16"])
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("n,V,F", [(60000, 3, 100), (262144, 50, 64), (262145, 50, 64), (700000, 20000, 36), (400000, 2, 130),
                                   (50000, 1700, 77)])
def test_table_gradient(G, n, V, F, kd, kt, add):
    """Normal values one by one: a chain of m has an error of U sqrt(m / 6) of its sum; chains of 32, and of 128 beyond
    2^18 places, in double. The sum, its product with the scale and, added, that with the table's value are
    each rounded to fp32: 3 U; bf16: half a step more."""
    import torch
    note("table gradient n=%d V=%d F=%d %s %s %s" % (n, V, F, kd, kt, add))
    gen = drawn(n + V)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}
    ids = (torch.rand(n, generator=gen, device="cuda:0") ** 2 * V).int().clamp(max=V - 1)
    dy = torch.randn(n, F, generator=gen, device="cuda:0").to(t[kd])
    old = torch.randn(V, F, generator=gen, device="cuda:0").to(t[kt])
    by, places, _ = G.gcn_group_ids(ids, V)
    dT = old.clone()
    G.gcn_embed_bwd(dy, by, places, scale=0.3, dT=dT, accumulate=add)
    want = torch.zeros(V, F, dtype=torch.float64, device="cuda:0").index_add_(0, ids.long(), dy.double())
    want = want * float(np.float32(0.3)) + (old.double() if add else 0)
    m = 32 if n <= 1 << 18 else 128
    bound = (3 + 2 * (m / 6) ** 0.5) * U + ref.HALF[kt]
    note("%.2f U of %.2f" % (off(dT, want) / U, bound / U))
    assert off(dT, want) <= bound


@pytest.mark.parametrize("n,V", [(2000, 9), (20000, 50), (300000, 200)])
def test_table_gradient_elements(G, n, V):
    """Every element within its chain's worst case: 31 or 127 additions, the roundings behind them."""
    import torch
    note("table gradient elements n=%d V=%d" % (n, V))
    gen, F = drawn(n), 40
    ids = (torch.rand(n, generator=gen, device="cuda:0") ** 2 * V).int().clamp(max=V - 1)
    dy = torch.randn(n, F, generator=gen, device="cuda:0")
    by, places, _ = G.gcn_group_ids(ids, V)
    got = G.gcn_embed_bwd(dy, by, places, scale=0.3).double()
    zero = torch.zeros(V, F, dtype=torch.float64, device="cuda:0")
    s = float(np.float32(0.3))
    want, mag = s * zero.index_add(0, ids.long(), dy.double()), s * zero.index_add(0, ids.long(), dy.double().abs())
    chain = 31 if n <= 1 << 18 else 127
    assert bool(((got - want).abs() <= chain * U * 1.001 * mag + 2.001 * U * want.abs() + 1e-37).all())
    assert np.isfinite(host(got)).all()
