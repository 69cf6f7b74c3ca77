"""INT8 linear layers on the GPU against their definition (tests/linear_ref.py):
integers and scales bit for bit, products against the exact sum.

Tolerance of a product: the INT32 sum is exact; its conversion to FP32, the
factors sa and sb and the bias are one rounding each, at most 2^-24 of the value
at that point, and the output's rounding is at most half a step of its type (and
half of the smallest subnormal).
"""
import numpy as np
import pytest
import torch

import linear_ref as ref
from gpu_helpers import DEV, note, to_dev
from paper_1802_00930_amd import dfp

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}
GUARD = 0x5a


def typed(a, t):
    """FP32 array rounded to a type: (device tensor, its values in FP32)."""
    x = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(TYPES[t])
    return x.to(DEV), x.float().numpy()


def check(got, y, size, t, what, roundings=4):
    got = got.float().cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(y)), what
    tol = roundings * 2.0 ** -24 * (size + np.abs(y)) + HALF_STEP[t] * np.abs(y) * (1 + 2.0 ** -20) + TINY[t]
    bad = np.abs(got - y) > tol
    assert not bad.any(), "%s: %d off, worst %g of the tolerance" % (
        what, bad.sum(), np.nanmax(np.abs(got - y) / tol))


def guarded(*shape, dtype=torch.int8):
    """A tensor with 256 guard bytes behind it, and a check that they are as they were."""
    n = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
    raw = torch.full((n + 256,), GUARD, dtype=torch.uint8, device=DEV)
    return raw[:n].view(dtype).view(*shape), lambda: bool((raw[n:] == GUARD).all())


def values(rng, rows, cols, spread=1.0):
    return (rng.standard_normal((rows, cols)) * np.exp(spread * rng.standard_normal((rows, 1)))).astype(np.float32)


QUANT_SHAPES = [(1, 1), (1, 3), (5, 7), (3, 127), (4, 128), (9, 129), (2, 512), (7, 513), (130, 1000), (3, 1025),
                (2, 2049), (3, 4097), (2, 8193), (2, 16384), (2, 16385), (300, 40)]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("rows,cols", QUANT_SHAPES)
def test_quantize_rows(rows, cols, t):
    note("quantize %dx%d %s" % (rows, cols, t))
    rng = np.random.default_rng(rows * 100003 + cols)
    x = values(rng, rows, cols)
    if rows > 2:
        x[1] = 0
    d, xf = typed(x, t)
    q, q_ok = guarded(rows, ref.ld(cols))
    qt, qt_ok = guarded(cols, ref.ld(rows))
    s, s_ok = guarded(rows, dtype=torch.float32)
    dfp.dfp_quantize_i8(d, q, s, qt)
    rq, rs = ref.quantize_rows(xf)
    assert np.array_equal(s.cpu().numpy(), rs)
    assert np.array_equal(q.cpu().numpy(), ref.padded(rq))
    assert np.array_equal(qt.cpu().numpy(), ref.padded(rq.T))
    assert q_ok() and qt_ok() and s_ok()


def test_quantize_ties_and_small_rows():
    ties = np.arange(-126.5, 127, 1, dtype=np.float32)  # s = 1: every value halfway
    rows = [np.append(ties, 127), np.append(ties * 3, 381),        # s = 3
            np.append(ties, 127) * np.float32(2.0 ** -120),        # s = 2^-120
            np.append(ties, 127) * np.float32(2.0 ** -140),        # subnormal numbers
            np.full(255, 2.0 ** -149, np.float32),                 # s rounds to 0
            np.append(np.zeros(254, np.float32), 190 * 2.0 ** -149),  # s = 2^-149: 190 is clamped to 127
            np.append(ties, 127) * np.float32(2.0 ** 120)]
    x = np.stack([r[:255] for r in rows]).astype(np.float32)
    d = to_dev(x)
    q = torch.empty(len(rows), ref.ld(255), dtype=torch.int8, device=DEV)
    s = torch.empty(len(rows), dtype=torch.float32, device=DEV)
    dfp.dfp_quantize_i8(d, q, s)
    rq, rs = ref.quantize_rows(x)
    assert rs[4] == 0 and rs[5] > 0 and rq[5].max() == 127
    assert np.array_equal(s.cpu().numpy(), rs)
    assert np.array_equal(q.cpu().numpy()[:, :255], rq)


def test_quantize_not_finite():
    rng = np.random.default_rng(5)
    x = values(rng, 6, 300)
    x[1, 7], x[3, 299], x[4, 0] = np.nan, np.inf, -np.inf
    q = torch.empty(6, ref.ld(300), dtype=torch.int8, device=DEV)
    s = torch.empty(6, dtype=torch.float32, device=DEV)
    dfp.dfp_quantize_i8(to_dev(x), q, s)
    rq, rs = ref.quantize_rows(x)
    assert np.isnan(rs[[1, 3, 4]]).all() and not np.isnan(rs[[0, 2, 5]]).any()
    assert np.array_equal(s.cpu().numpy(), rs, equal_nan=True)
    assert np.array_equal(q.cpu().numpy()[:, :300], rq)


@pytest.mark.parametrize("rows,cols", [(3, 5), (4, 130), (2, 1030), (1, 2051)])
def test_quantize_stochastic(rows, cols):
    rng = np.random.default_rng(cols)
    x = values(rng, rows, cols)
    seed, role = 0x1234567890abcdef, dfp.ROLE_W
    q = torch.empty(rows, ref.ld(cols), dtype=torch.int8, device=DEV)
    s = torch.empty(rows, dtype=torch.float32, device=DEV)
    dfp.dfp_quantize_i8(to_dev(x), q, s, rounding="stochastic", seed=seed, role=role)
    rq, rs = ref.quantize_rows(x, "stochastic", seed, role)
    assert np.array_equal(s.cpu().numpy(), rs)
    assert np.array_equal(q.cpu().numpy(), ref.padded(rq))
    assert not np.array_equal(rq, ref.quantize_rows(x)[0])


PRODUCTS = [(1, 1, 1), (1, 7, 130), (1, 130, 2049), (2, 16, 64), (3, 5, 127), (5, 1000, 257), (8, 64, 4096),
            (15, 33, 500), (16, 48, 1024), (17, 129, 640), (31, 64, 1500), (33, 100, 3000), (64, 1000, 2048),
            (65, 15, 300), (100, 300, 128), (127, 129, 255), (128, 128, 512), (130, 260, 1111), (257, 513, 200),
            (300, 1, 77), (1000, 40, 90), (700, 900, 33), (256, 512, 1024), (1025, 1030, 160)]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, t):
    note("product %dx%dx%d %s" % (m, n, k, t))
    rng = np.random.default_rng(m * 7919 + n * 31 + k)
    a, b = (rng.integers(-128, 128, s).astype(np.int8) for s in ((m, k), (n, k)))
    sa, sb = (np.exp(rng.standard_normal(s)).astype(np.float32) * 2.0 ** -9 for s in (m, n))
    bias = rng.standard_normal(n).astype(np.float32) if (m + n + k) % 2 else None
    d = dfp.make_linear_desc(m, n, k, TYPES[t])
    out, ok = guarded(m, n, dtype=TYPES[t])
    ta, tb = to_dev(ref.padded(a)), to_dev(ref.padded(b))
    ws = dfp.alloc_linear_i8_workspace(d)
    for _ in range(2):
        dfp.dfp_gemm_i8(d, ta, to_dev(sa), tb, to_dev(sb), out, bias=None if bias is None else to_dev(bias),
                        workspace=ws)
    y, size = ref.product(a, sa, b, sb, bias)
    check(out, y, size, t, "product %dx%dx%d" % (m, n, k))
    assert ok()


@pytest.mark.parametrize("m", [2, 40, 200])
def test_product_at_the_longest_sum(m):
    """131071 products of (-128)^2 stay below 2^31."""
    k, n = dfp.lib() and 131071, 3
    a = torch.zeros(m, ref.ld(k), dtype=torch.int8, device=DEV)
    b = torch.zeros(n, ref.ld(k), dtype=torch.int8, device=DEV)
    a[:, :k], b[:, :k] = -128, -128
    b[1] = -b[1] - 1  # 127
    b[1, k:] = 0
    one = torch.ones(max(m, n), device=DEV)
    out = torch.empty(m, n, device=DEV)
    d = dfp.make_linear_desc(m, n, k, torch.float32)
    dfp.dfp_gemm_i8(d, a, one[:m].clone(), b, one[:n].clone(), out, workspace=dfp.alloc_linear_i8_workspace(d))
    want = np.tile(np.array([128 * 128 * k, -128 * 127 * k, 128 * 128 * k], np.int64).astype(np.float32), (m, 1))
    assert np.array_equal(out.cpu().numpy(), want)


class Layer:
    """A layer's inputs on both sides and its calls."""

    def __init__(self, m, n, k, t, bias=True, rounding="nearest", seed=0, zero_rows=True):
        rng = np.random.default_rng(m * 1009 + n * 13 + k)
        self.m, self.n, self.k, self.t, self.rounding, self.seed = m, n, k, t, rounding, seed
        self.w = (rng.standard_normal((n, k)) * np.sqrt(2 / k)).astype(np.float32)
        x, dy = values(rng, m, k, 0.5), values(rng, m, n)
        if zero_rows and m > 3:
            x[1], dy[2] = 0, 0
        if zero_rows and n > 3:
            dy[:, 3] = 0
        self.tx, self.x = typed(x, t)
        self.tdy, self.dy = typed(dy, t)
        self.bias = rng.standard_normal(n).astype(np.float32) if bias else None
        self.wq, self.sw = ref.quantize_rows(self.w)
        self.twq, self.twqt, self.tsw = to_dev(ref.padded(self.wq)), to_dev(ref.padded(self.wq.T)), to_dev(self.sw)
        self.tb = to_dev(self.bias) if bias else None
        self.d = dfp.make_linear_desc(m, n, k, TYPES[t], rounding=rounding, seed=seed)
        self.ws = torch.full((dfp.linear_i8_workspace_bytes(self.d),), 0xff, dtype=torch.uint8, device=DEV)
        T = TYPES[t]
        self.y, self.dx = (torch.empty(m, c, dtype=T, device=DEV) for c in (n, k))
        self.dw, self.db = torch.empty(n, k, device=DEV), torch.empty(n, device=DEV)
        self.xq = torch.empty(m, ref.ld(k), dtype=torch.int8, device=DEV)
        self.xqt = torch.empty(k, ref.ld(m), dtype=torch.int8, device=DEV)
        self.sx = torch.empty(m, device=DEV)

    def run(self, stream=None):
        dfp.dfp_linear_i8_fwd(self.d, self.tx, self.twq, self.tsw, self.y, bias=self.tb, xq=self.xq, sx=self.sx,
                              xqt=self.xqt, workspace=self.ws, stream=stream)
        dfp.dfp_linear_i8_bwd_data(self.d, self.tdy, self.twqt, self.tsw, self.dx, workspace=self.ws, stream=stream)
        dfp.dfp_linear_i8_bwd_weights(self.d, self.tdy, self.xqt, self.sx, self.dw, db=self.db, workspace=self.ws,
                                      stream=stream)

    def check(self):
        what = "%dx%dx%d %s" % (self.m, self.n, self.k, self.t)
        xq, sx = ref.quantize_rows(self.x, self.rounding, self.seed, dfp.ROLE_X)
        assert np.array_equal(self.xq.cpu().numpy(), ref.padded(xq)), what
        assert np.array_equal(self.xqt.cpu().numpy(), ref.padded(xq.T)), what
        assert np.array_equal(self.sx.cpu().numpy(), sx, equal_nan=True), what
        check(self.y, *ref.product(xq, sx, self.wq, self.sw, self.bias), self.t, what + " y")
        # a product of two FP32 numbers is exact in 64 bits: one rounding
        g = (self.dy.astype(np.float64) * self.sw[None, :]).astype(np.float32)
        gq, sg = ref.quantize_rows(g, self.rounding, self.seed, dfp.ROLE_DY)
        check(self.dx, *ref.product(gq, sg, self.wq.T), self.t, what + " dx")
        g = (self.dy.astype(np.float64) * sx[:, None]).astype(np.float32)
        order = np.arange(g.size).reshape(g.shape).T
        gq, sg = ref.quantize_rows(g.T, self.rounding, self.seed, dfp.ROLE_DY, order)
        check(self.dw, *ref.product(gq, sg, xq.T), "f32", what + " dw")
        # at most m + 16 additions, each off by 2^-24 of a partial sum of absolute values
        total = np.abs(self.dy.astype(np.float64)).sum(0)
        err = np.abs(self.db.cpu().numpy() - self.dy.astype(np.float64).sum(0))
        assert (err <= (self.m + 16) * 2.0 ** -24 * total).all(), what


LAYERS = [(1, 1, 1), (1, 40, 70), (2, 3, 200), (7, 130, 129), (16, 64, 256), (33, 200, 100), (63, 257, 130),
          (129, 65, 127), (200, 128, 128), (500, 300, 77), (1000, 33, 260), (4097, 20, 12)]


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,n,k", LAYERS)
def test_layer(m, n, k, t):
    note("layer %dx%dx%d %s" % (m, n, k, t))
    layer = Layer(m, n, k, t, bias=m % 2 == 1)
    layer.run()
    layer.check()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(131071, 3, 2), (30001, 65, 10), (33, 70000, 3), (1025, 4100, 5)])
def test_long_and_wide_gradients(m, n, k, t):
    """Columns whose maxima and sums come from many slices of the tokens, or from one."""
    note("layer %dx%dx%d %s" % (m, n, k, t))
    layer = Layer(m, n, k, t)
    layer.run()
    layer.check()


@pytest.mark.parametrize("m,n,k", [(3, 5, 9), (20, 130, 33)])
def test_layer_stochastic(m, n, k):
    layer = Layer(m, n, k, "bf16", rounding="stochastic", seed=99)
    layer.run()
    layer.check()


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("m,k", [(1, 1), (1, 300), (2, 77), (2, 300), (1, 4097), (2, 8200), (1, 20001), (1, 40000),
                                 (2, 20001), (3, 300)])
def test_few_tokens(m, k, t, rounding):
    """One or two tokens run in one launch, which quantises them as the other calls do."""
    layer = Layer(m, 50, k, t, rounding=rounding, seed=7, zero_rows=False)
    if m == 2:
        layer.tx[1] = 0
        layer.x[1] = 0
    layer.run()
    y = torch.empty_like(layer.y)
    dfp.dfp_linear_i8_fwd(layer.d, layer.tx, layer.twq, layer.tsw, y, bias=layer.tb, workspace=layer.ws)
    assert torch.equal(y.float(), layer.y.float())
    layer.tx[0, k // 2] = float("nan")
    dfp.dfp_linear_i8_fwd(layer.d, layer.tx, layer.twq, layer.tsw, y, bias=layer.tb, workspace=layer.ws)
    assert torch.isnan(y[0]).all() and torch.equal(y[1:].float(), layer.y[1:].float())


@pytest.mark.parametrize("m", [1, 6, 40, 300])
def test_forward_without_saved_tensors(m):
    layer = Layer(m, 70, 300, "bf16")
    layer.run()
    y = torch.empty_like(layer.y)
    dfp.dfp_linear_i8_fwd(layer.d, layer.tx, layer.twq, layer.tsw, y, bias=layer.tb, workspace=layer.ws)
    assert torch.equal(y.view(torch.int16), layer.y.view(torch.int16))
    dw = torch.empty_like(layer.dw)
    dfp.dfp_linear_i8_bwd_weights(layer.d, layer.tdy, layer.xqt, layer.sx, dw, workspace=layer.ws)
    assert torch.equal(dw, layer.dw)


@pytest.mark.parametrize("m", [3, 50])
def test_a_token_that_is_not_finite(m):
    layer = Layer(m, 40, 60, "f32", zero_rows=False)
    layer.x[1, 5] = np.nan
    layer.tx = to_dev(layer.x)
    layer.run()
    layer.check()  # its row of y is NaN, and all of dw
    assert torch.isnan(layer.y[1]).all() and not torch.isnan(layer.y[0]).any() and torch.isnan(layer.dw).all()


def test_gradients_against_differences():
    """Integers that quantise to themselves (every row and column holds a 127, scales
    powers of two) make the layer linear: its gradients are differences of y."""
    rng = np.random.default_rng(11)
    m, n, k = 9, 20, 30
    x, w, dy = (rng.integers(-126, 126, s).astype(np.float32) for s in ((m, k), (n, k), (m, n)))
    x[:, 0], w[:, 0], dy[:, 0], dy[0, :] = 127, 127, 127, 127
    layer = Layer(m, n, k, "f32", bias=False)
    layer.wq, layer.sw = ref.quantize_rows(w)
    layer.x, layer.dy = x, dy
    layer.tx, layer.tdy = to_dev(x), to_dev(dy)
    layer.twq, layer.twqt, layer.tsw = to_dev(ref.padded(layer.wq)), to_dev(ref.padded(layer.wq.T)), to_dev(layer.sw)
    layer.run()
    y0 = layer.y.cpu().numpy().astype(np.float64)
    dx, dw = layer.dx.cpu().numpy(), layer.dw.cpu().numpy()
    assert np.array_equal(y0, x.astype(np.float64) @ w.T.astype(np.float64))
    for j in (1, 7, k - 1):
        layer.tx = to_dev(x + np.eye(k, dtype=np.float32)[j][None, :])
        layer.run()
        diff = ((layer.y.cpu().numpy() - y0) * dy).sum(1)
        assert np.array_equal(diff, dx[:, j].astype(np.float64))
    layer.tx = to_dev(x)
    for i, j in ((0, 1), (5, 17), (n - 1, k - 1)):
        w1 = w.copy()
        w1[i, j] += 1
        layer.twq = to_dev(ref.padded(ref.quantize_rows(w1)[0]))
        layer.run()
        assert ((layer.y.cpu().numpy() - y0) * dy).sum() == dw[i, j]


@pytest.mark.parametrize("m", [1, 24, 200])
def test_captured_and_on_another_stream(m):
    """Captured once and replayed beside eager work on new inputs, every replay as the eager call."""
    layer, other = Layer(m, 130, 200, "bf16"), Layer(m, 70, 300, "bf16")
    layer.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        layer.run()
        with torch.cuda.graph(g, stream=side):
            layer.run()
    torch.cuda.synchronize()
    rng = np.random.default_rng(3)
    for i in range(3):
        x, dy = values(rng, m, 200), values(rng, m, 130)
        layer.tx.copy_(to_dev(x)), layer.tdy.copy_(to_dev(dy))
        layer.x, layer.dy = layer.tx.float().cpu().numpy(), layer.tdy.float().cpu().numpy()
        for out in (layer.y, layer.dx, layer.dw, layer.db):
            out.zero_()
        g.replay()
        other.run()
        torch.cuda.synchronize()
        layer.check()
        other.check()


def test_two_calls_at_once():
    a, b = Layer(300, 200, 500, "bf16"), Layer(300, 200, 500, "f32", bias=False)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(4):
        a.run(stream=s1)
        b.run(stream=s2)
    torch.cuda.synchronize()
    a.check()
    b.check()


def test_binding_refuses():
    layer = Layer(4, 8, 16, "f32")
    with pytest.raises(ValueError):
        dfp.dfp_linear_i8_fwd(layer.d, layer.tx[:3].contiguous(), layer.twq, layer.tsw, layer.y, workspace=layer.ws)
    with pytest.raises(TypeError):
        dfp.dfp_linear_i8_fwd(layer.d, layer.tx.double(), layer.twq, layer.tsw, layer.y, workspace=layer.ws)
    with pytest.raises(TypeError):
        dfp.dfp_linear_i8_fwd(layer.d, layer.tx.t().contiguous().t(), layer.twq, layer.tsw, layer.y,
                              workspace=layer.ws)
    with pytest.raises(TypeError):
        dfp.dfp_linear_i8_fwd(layer.d, layer.tx.cpu(), layer.twq, layer.tsw, layer.y, workspace=layer.ws)
    with pytest.raises(dfp.DfpError):
        dfp.dfp_linear_i8_fwd(layer.d, layer.tx, layer.twq, layer.tsw, layer.y)
    with pytest.raises(ValueError):
        dfp.dfp_quantize_i8(layer.tx, layer.twq, layer.sx)
