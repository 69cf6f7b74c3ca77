"""Stochastic rounding of the INT8 calls at rows of every length that has a form of its own, all types, bit for bit
against the definition; rows and columns of zeros among them, as masked tokens leave in a gradient."""
import numpy as np
import pytest
import torch

import linear_ref as ref
import test_gpu_linear_i8 as layers
from gpu_helpers import DEV, note
from paper_1802_00930_amd import dfp

pytestmark = pytest.mark.gpu
SEED = 0xfedcba9876543210


@pytest.mark.parametrize("t", list(layers.TYPES))
@pytest.mark.parametrize("rows,cols", [(3, 601), (2, 1003), (514, 1100), (3, 2048), (2, 4001), (2, 8004), (1, 16384),
                                       (1, 20002)])
def test_quantize(rows, cols, t):
    note("stochastic %dx%d %s" % (rows, cols, t))
    x = layers.values(np.random.default_rng(rows + cols), rows, cols)
    x[rows // 2] = 0 if rows > 1 else x[rows // 2]
    d, xf = layers.typed(x, t)
    q, q_ok = layers.guarded(rows, ref.ld(cols))
    s = torch.empty(rows, device=DEV)
    dfp.dfp_quantize_i8(d, q, s, rounding="stochastic", seed=SEED, role=dfp.ROLE_DY)
    rq, rs = ref.quantize_rows(xf, "stochastic", SEED, dfp.ROLE_DY)
    assert np.array_equal(s.cpu().numpy(), rs) and np.array_equal(q.cpu().numpy(), ref.padded(rq)) and q_ok()


@pytest.mark.parametrize("t", list(layers.TYPES))
@pytest.mark.parametrize("m,n,k", [(1, 130, 600), (140, 70, 129), (33, 1100, 40)])
def test_layer(m, n, k, t):
    """Zero rows of x and dy, and a zero column of dy."""
    note("stochastic layer %dx%dx%d %s" % (m, n, k, t))
    layer = layers.Layer(m, n, k, t, rounding="stochastic", seed=SEED)
    layer.run()
    layer.check()


@pytest.mark.parametrize("m,k", [(1, 700), (2, 9001), (1, 32768)])
def test_tokens(m, k):
    note("stochastic tokens %dx%d" % (m, k))
    layer = layers.Layer(m, 40, k, "bf16", rounding="stochastic", seed=SEED)
    dfp.dfp_linear_i8_fwd(layer.d, layer.tx, layer.twq, layer.tsw, layer.y, bias=layer.tb, workspace=layer.ws)
    xq, sx = ref.quantize_rows(layer.x, "stochastic", SEED, dfp.ROLE_X)
    layers.check(layer.y, *ref.product(xq, sx, layer.wq, layer.sw, layer.bias), "bf16", "y")


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
def test_masked_tokens(rounding):
    """Half of the tokens are masked: their rows of dy are zeros, their rows of dx too, and dw is that of the rest."""
    layer = layers.Layer(96, 50, 140, "bf16", rounding=rounding, seed=SEED, zero_rows=False)
    layer.tdy[::2] = 0
    layer.dy[::2] = 0
    layer.run()
    layer.check()
    assert not layer.dx[::2].any() and layer.dx[1::2].any()
