"""INT8 linear layers and orthogonalised updates on tensors whose offsets pass 32 bits (2^31 and 2^32 elements, the
Philox counter 2^32), against their definition on the GPU or, for single rows, in NumPy.  Tolerances as in
test_gpu_linear_i8.py and test_gpu_ortho.py.  Up to 120 GB of the card."""
import numpy as np
import pytest
import torch

import linear_ref as ref
from gpu_helpers import DEV, note
from paper_1802_00930_amd import dfp

pytestmark = pytest.mark.gpu
CHUNK = 2048


@pytest.fixture(autouse=True)
def _room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 140 << 30:
        pytest.skip("less than 140 GB free")
    yield
    torch.cuda.empty_cache()


def generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(seed, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=generator(seed), device=DEV, dtype=dtype)


def integers(seed, rows, cols):
    q = torch.zeros(rows, ref.ld(cols), dtype=torch.int8, device=DEV)
    q[:, :cols] = torch.randint(-127, 128, (rows, cols), generator=generator(seed), device=DEV, dtype=torch.int8)
    return q


def quantised(x):
    """(integers as FP64, scales) of the rows of FP32 values."""
    s = (x.abs().amax(1).double() / 127).float()
    return torch.round(x.double() / s.double()[:, None]).clamp_(-127, 127), s


def chunks(n):
    return [slice(i, min(n, i + CHUNK)) for i in range(0, n, CHUNK)]


def near(got, y, size, half):
    return bool(((got.double() - y).abs() <= 4 * 2.0 ** -24 * (size + y.abs()) + half * 1.0001 * y.abs()).all())


def test_quantize():
    rows, cols = 65700, 65600
    note("quantise %dx%d" % (rows, cols))
    x = normal(1, rows, cols, dtype=torch.bfloat16)
    q = torch.full((rows, ref.ld(cols)), 99, dtype=torch.int8, device=DEV)
    qt = torch.full((cols, ref.ld(rows)), 99, dtype=torch.int8, device=DEV)
    s = torch.empty(rows, device=DEV)
    dfp.dfp_quantize_i8(x, q, s, qt)
    for c in chunks(rows):
        want, scale = quantised(x[c].float())
        assert torch.equal(s[c], scale), c
        assert torch.equal(q[c, :cols], want.to(torch.int8)) and not q[c, cols:].any(), c
    for c in chunks(cols):
        assert torch.equal(qt[c, :rows], q[:, c].t()) and not qt[c, rows:].any(), c


def test_quantize_stochastic():
    """Row 131072 begins at flat index 2^34, whose Philox counter is 2^32."""
    rows, cols = 131080, 131072
    note("quantise %dx%d, stochastic" % (rows, cols))
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device=DEV)
    some = [0, 1, 131071, 131072, 131079]
    for r in some:
        x[r].copy_(normal(r, cols, dtype=torch.bfloat16))
    q = torch.full((rows, cols), 99, dtype=torch.int8, device=DEV)
    s = torch.empty(rows, device=DEV)
    dfp.dfp_quantize_i8(x, q, s, rounding="stochastic", seed=77, role=dfp.ROLE_W)
    for r in some:
        order = np.arange(cols, dtype=np.int64)[None] + r * cols
        rq, rs = ref.quantize_rows(x[r:r + 1].float().cpu().numpy(), "stochastic", 77, dfp.ROLE_W, order)
        assert np.array_equal(q[r].cpu().numpy(), rq[0]) and float(s[r]) == rs[0], r
    s[some] = 0
    assert not s.any()
    for c in chunks(131071):
        if c.start > 1:
            assert not q[c.start:min(c.stop, 131071)].any(), c


def test_layer():
    m, n, k = 65700, 65600, 96
    note("layer %dx%dx%d" % (m, n, k))
    wq = integers(3, n, k)
    wqt = torch.zeros(k, ref.ld(n), dtype=torch.int8, device=DEV)
    wqt[:, :n] = wq[:, :k].t()
    sw = torch.rand(n, generator=generator(4), device=DEV) * 2.0 ** -8 + 2.0 ** -10
    bias = normal(5, n)
    x, dy = normal(6, m, k, dtype=torch.bfloat16), normal(7, m, n, dtype=torch.bfloat16)
    d = dfp.make_linear_desc(m, n, k, torch.bfloat16)
    ws = dfp.alloc_linear_i8_workspace(d)
    y, dx = torch.empty(m, n, dtype=torch.bfloat16, device=DEV), torch.empty_like(x)
    dw, db, sx = torch.empty(n, k, device=DEV), torch.empty(n, device=DEV), torch.empty(m, device=DEV)
    xqt = torch.empty(k, ref.ld(m), dtype=torch.int8, device=DEV)
    dfp.dfp_linear_i8_fwd(d, x, wq, sw, y, bias=bias, sx=sx, xqt=xqt, workspace=ws)
    xq, scale = quantised(x.float())
    assert torch.equal(sx, scale) and torch.equal(xqt[:, :m], xq.t().to(torch.int8))
    w64, b64 = wq[:, :k].double(), bias.double()[None]
    for c in chunks(m):
        want = torch.mm(xq[c], w64.t()) * sx[c].double()[:, None] * sw.double()[None]
        assert near(y[c], want + b64, want.abs(), 2.0 ** -8), c
    del y
    dfp.dfp_linear_i8_bwd_data(d, dy, wqt, sw, dx, workspace=ws)
    for c in chunks(m):
        gq, sg = quantised(dy[c].float() * sw[None])
        want = torch.mm(gq, w64) * sg.double()[:, None]
        assert near(dx[c], want, want.abs(), 2.0 ** -8), c
    dfp.dfp_linear_i8_bwd_weights(d, dy, xqt, sx, dw, db=db, workspace=ws)
    for c in chunks(n):
        part = dy[:, c].float()
        gq, sg = quantised((part * sx[:, None]).t().contiguous())
        want = torch.mm(gq, xq) * sg.double()[:, None]
        assert near(dw[c], want, want.abs(), 2.0 ** -24), c
        off = (db[c].double() - part.double().sum(0)).abs()
        assert bool((off <= (m + 16) * 2.0 ** -24 * part.double().abs().sum(0)).all()), c


@pytest.mark.parametrize("m", [1, 3, 20, 200])
def test_long_operand(m):
    """The long operand as weights, and as activations."""
    n, k = 140000, 32700
    note("product %dx%dx%d and its transpose" % (m, n, k))
    a, b = integers(8, m, k), integers(9, n, k)
    sa, sb = (torch.rand(r, generator=generator(r), device=DEV) * 2.0 ** -6 for r in (m, n))
    out, outt = torch.empty(m, n, device=DEV), torch.empty(n, m, device=DEV)
    d, dt = dfp.make_linear_desc(m, n, k, torch.float32), dfp.make_linear_desc(n, m, k, torch.float32)
    dfp.dfp_gemm_i8(d, a, sa, b, sb, out, workspace=dfp.alloc_linear_i8_workspace(d))
    dfp.dfp_gemm_i8(dt, b, sb, a, sa, outt, workspace=dfp.alloc_linear_i8_workspace(dt))
    a64 = a.double()
    for c in chunks(n):
        want = torch.mm(a64, b[c].double().t()) * sa.double()[:, None] * sb[c].double()[None]
        assert near(out[:, c], want, want.abs(), 2.0 ** -24), c
        assert near(outt[c], want.t(), want.t().abs(), 2.0 ** -24), c
    if m == 1:  # the forward call of one token reads the same weights in its own kernel
        x = a[:, :k].float()
        x[0, 0] = 127
        y = torch.empty(1, n, device=DEV)
        dfp.dfp_linear_i8_fwd(d, x, b, sb, y, workspace=dfp.alloc_linear_i8_workspace(d))
        for c in chunks(n):
            want = torch.mm(x.double(), b[c, :k].double().t()) * sb[c].double()[None]
            assert near(y[:, c], want, want.abs(), 2.0 ** -24), c


def newton_schulz(u):
    x = u.double() / (torch.linalg.vector_norm(u.double()) + 1e-7)
    for _ in range(5):
        g = torch.mm(x, x.t().contiguous())
        x = 3.4445 * x + torch.mm(-4.7750 * g + 2.0315 * torch.mm(g, g), x)
    return x


BATCH, R, C = 16400, 64, 4096  # matrix 8192 begins at element 2^31, 16384 at 2^32
SOME = [0, 8191, 8192, 16383, 16384, 16399]


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
def test_orthogonalize(t):
    note("orthogonalise %dx%dx%d %s" % (BATCH, R, C, t))
    x = normal(11, BATCH, R, C, dtype=t)
    before = [x[i].clone() for i in SOME]
    d = dfp.make_ortho_desc(BATCH, R, C, t)
    dfp.dfp_orthogonalize(d, x, x, workspace=dfp.alloc_ortho_workspace(d))
    for i, u in zip(SOME, before):
        want = newton_schulz(u)
        off = float(torch.linalg.vector_norm(x[i].double() - want) / torch.linalg.vector_norm(want))
        assert off <= (2e-4 if t is torch.float32 else 3e-3), (i, off)


def test_weight_step():
    note("weight step %dx%dx%d" % (BATCH, R, C))
    w, v, dw = normal(12, BATCH, R, C), torch.zeros(BATCH, R, C, device=DEV), normal(13, BATCH, R, C)
    before = [w[i].clone() for i in SOME]
    d = dfp.make_ortho_desc(BATCH, R, C, torch.float32)
    wq = torch.empty(BATCH * R, C, dtype=torch.int8, device=DEV)
    sw = torch.empty(BATCH * R, device=DEV)
    dfp.dfp_muon_quantize(d, 1.0, 0.5, 0.1, 0.5, w, v, dw, wq, sw, nesterov=False,
                          workspace=dfp.alloc_ortho_workspace(d))
    for i, old in zip(SOME, before):
        assert torch.equal(v[i], dw[i])
        step = 0.5 * newton_schulz(dw[i])
        want = float(np.float32(0.9)) * old.double() - step
        off = float(torch.linalg.vector_norm(w[i].double() - want))
        # O's tolerance, 3e-4 where iterations are taken together, and w's own roundings
        assert off <= 3e-4 * float(torch.linalg.vector_norm(step)) + 4 * 2.0 ** -24 * float(torch.linalg.vector_norm(want)), i
        q, s = quantised(w[i])
        rows = slice(i * R, (i + 1) * R)
        assert torch.equal(sw[rows], s) and torch.equal(wq[rows], q.to(torch.int8)), i
