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
