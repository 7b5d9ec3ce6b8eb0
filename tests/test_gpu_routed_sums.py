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


def off(got, want):
    """The error in the matrix's norm."""
    return float((got.double() - want).norm() / want.norm())


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
