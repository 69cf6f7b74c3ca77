"""Orthogonalised updates on the GPU against the iteration in 64 bits.

Tolerances, in the norm of the result.  FP32 and F16 results: an operand as two
f16 numbers is off by 2^-22 of its value and a product leaves out 2^-22, so a step
adds at most about 2^-20 of X; the steps after it multiply the smallest singular
values' share by up to a each: 2^-20 (1 + 3.45 + ... + 3.45^4) = 2e-4.  BF16
results: the products on single f16 numbers are documented to stay under half of
BF16's half step, 2^-9, and the result's own rounding adds 2^-8 / sqrt(3) at most
(uniform within a step): 3e-3 together.  That mean is one over many elements: the
rounding of each may take up all of 2^-8 of it (0.5606 to 0.5625), and of a matrix
of a few elements so may the norm's, which allows 2^-9 + 2^-8 there.  F16 results:
as FP32 plus 2^-11.
"""
import numpy as np
import pytest
import torch

import linear_ref as ref
from gpu_helpers import DEV, note, to_dev
from paper_1802_00930_amd import dfp

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TOL = {"f32": 2e-4, "bf16": 3e-3, "f16": 2e-4 + 2.0 ** -11}
COEF = (3.4445, -4.7750, 2.0315)


def matrices(rng, b, r, c, kind):
    u = rng.standard_normal((b, r, c)) * np.exp(0.5 * rng.standard_normal((b, r, 1)))
    if kind == "low_rank":
        k = max(1, min(r, c) // 16)
        u = 0.2 * u + rng.standard_normal((b, r, k)) @ rng.standard_normal((b, k, c))
    return (1e-3 * u).astype(np.float32)


def run(x, t, steps=5, coef=COEF, eps=1e-7, alias=False, garbage=0xff):
    b, r, c = x.shape
    tx = torch.from_numpy(x).to(TYPES[t]).to(DEV)
    d = dfp.make_ortho_desc(b, r, c, TYPES[t], steps=steps, eps=eps, coef=coef)
    ws = torch.full((dfp.ortho_workspace_bytes(d),), garbage, dtype=torch.uint8, device=DEV)
    out = tx if alias else torch.full_like(tx, 7.0)
    xf = tx.float().cpu().numpy()
    dfp.dfp_orthogonalize(d, tx, out, workspace=ws)
    return out.float().cpu().numpy(), xf


def assert_near(got, want, tol, what):
    if tol == TOL["bf16"] and want.size < 64:
        tol = 2.0 ** -9 + 2.0 ** -8
    norm = np.linalg.norm(want)
    assert np.isfinite(got).all(), what
    assert np.linalg.norm(got - want) <= tol * norm, "%s: %g of the tolerance" % (
        what, np.linalg.norm(got - want) / norm / tol)


SHAPES = [(1, 1, 1), (1, 1, 7), (2, 5, 1), (3, 2, 2), (1, 64, 64), (2, 100, 260), (1, 333, 130), (3, 129, 128),
          (1, 128, 129), (1, 17, 700), (1, 700, 17), (1, 256, 256), (2, 257, 300), (1, 300, 520)]


@pytest.mark.parametrize("kind", ["full", "low_rank"])
@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("b,r,c", SHAPES)
def test_orthogonalize(b, r, c, t, kind):
    note("ortho %dx%dx%d %s %s" % (b, r, c, t, kind))
    x = matrices(np.random.default_rng(b * 31 + r * 7 + c), b, r, c, kind)
    got, xf = run(x, t)
    for i in range(b):
        want = ref.newton_schulz(xf[i], [COEF] * 5, np.float32(1e-7))
        assert_near(got[i], want, TOL[t], "%s %s matrix %d" % (t, kind, i))


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("r,c", [(60, 200), (200, 60)])
def test_singular_values_near_one(r, c, t):
    """Coefficients whose fixed point is 1: the result has orthonormal rows or columns."""
    x = matrices(np.random.default_rng(1), 1, r, c, "full")
    coef = [(4.0, -6.0, 2.6)] * 2 + [(15 / 8, -10 / 8, 3 / 8)] * 8
    got, xf = run(x, t, steps=10, coef=coef)
    want = ref.newton_schulz(xf[0], coef, np.float32(1e-7))
    assert_near(got[0], want, 2 * TOL[t], t)
    assert np.linalg.svd(got[0], compute_uv=False).max() < 1.02


def test_one_step_and_in_place():
    x = matrices(np.random.default_rng(2), 2, 40, 90, "full")
    for t in TYPES:
        got, xf = run(x, t, steps=1, coef=(1.5, -0.5, 0.0))
        again, _ = run(x, t, steps=1, coef=(1.5, -0.5, 0.0), alias=True, garbage=0)
        assert np.array_equal(got, again)
        for i in range(2):
            assert_near(got[i], ref.newton_schulz(xf[i], [(1.5, -0.5, 0.0)], np.float32(1e-7)), TOL[t], t)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_zero_and_not_finite_matrices_of_a_batch(t):
    x = matrices(np.random.default_rng(3), 5, 30, 50, "full")
    x[1], x[2, 3, 4], x[3, 29, 49] = 0, np.nan, np.inf
    got, xf = run(x, t)
    assert (got[1] == 0).all() and np.isnan(got[2]).all() and np.isnan(got[3]).all()
    for i in (0, 4):
        assert_near(got[i], ref.newton_schulz(xf[i], [COEF] * 5, np.float32(1e-7)), TOL[t], t)


@pytest.mark.parametrize("r,c", [(256, 256), (300, 700), (700, 300)])
def test_strong_directions_above_weak_ones(r, c):
    """FP32 results are as near as FP32 products bring them: at most twice as far from
    64 bits as the same iteration in FP32 (an operand of two f16 numbers carries 2^-23
    of a value, FP32 2^-24)."""
    rng = np.random.default_rng(6)
    x = 0.1 * rng.standard_normal((r, c)) * np.exp(rng.standard_normal((r, 1)))
    x = (x + rng.standard_normal((r, 32)) @ rng.standard_normal((32, c)))[None].astype(np.float32)
    got, xf = run(x, "f32")
    want = ref.newton_schulz(xf[0], [COEF] * 5, np.float32(1e-7))
    u = torch.from_numpy(xf[0] if r <= c else np.ascontiguousarray(xf[0].T))
    u = (u.double() / (u.double().norm() + 1e-7)).float()
    for _ in range(5):
        a = u @ u.T
        u = COEF[0] * u + (COEF[1] * a + COEF[2] * (a @ a)) @ u
    plain = u.numpy() if r <= c else u.numpy().T
    off = [np.linalg.norm(y - want) / np.linalg.norm(want) for y in (got[0], plain)]
    assert off[0] <= 2 * off[1], off


@pytest.mark.parametrize("scale", [1e-30, 1e-4, 1e15, 1e33])
def test_magnitudes(scale):
    """The norm is taken in 64 bits: squares neither overflow nor vanish."""
    x = (1e3 * matrices(np.random.default_rng(4), 1, 48, 80, "full")) * np.float32(scale)
    eps = 1e-7 if scale > 1e-10 else 1e-37
    got, xf = run(x.astype(np.float32), "f32", eps=eps)
    assert_near(got[0], ref.newton_schulz(xf[0], [COEF] * 5, np.float32(eps)), TOL["f32"], str(scale))


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("b,r,c", [(1, 1, 5), (1, 96, 200), (1, 200, 96), (2, 130, 131), (1, 33, 1100)])
def test_muon_two_steps(b, r, c, t, nesterov):
    note("muon %dx%dx%d %s %d" % (b, r, c, t, nesterov))
    rng = np.random.default_rng(r * 3 + c)
    lr, mu, wd, scale = 0.02, 0.95, 0.1, 0.5
    w, v = (0.02 * rng.standard_normal((b, r, c))).astype(np.float32), matrices(rng, b, r, c, "low_rank")
    d = dfp.make_ortho_desc(b, r, c, TYPES[t])
    tw, tv, ws = to_dev(w), to_dev(v), dfp.alloc_ortho_workspace(d)
    wq = torch.empty(b * r, ref.ld(c), dtype=torch.int8, device=DEV)
    sw = torch.empty(b * r, device=DEV)
    wqt = torch.empty(c, ref.ld(r), dtype=torch.int8, device=DEV) if b == 1 else None
    w64, v64 = w.astype(np.float64), v.astype(np.float64)
    for step in range(2):
        g = torch.from_numpy(matrices(rng, b, r, c, "full")).to(TYPES[t])
        dfp.dfp_muon_quantize(d, lr, mu, wd, scale, tw, tv, g.to(DEV), wq, sw, wqt, nesterov=nesterov, workspace=ws)
        g64 = g.double().numpy()
        v64 = mu * v64 + g64
        u = g64 + mu * v64 if nesterov else v64
        o = np.stack([ref.newton_schulz(m, [COEF] * 5, 1e-7) for m in u])
        w64 = (1 - lr * wd) * w64 - lr * scale * o
        # v: the rounding of mu and of each fma; w: O's tolerance and its own roundings, over the steps so far
        dv = np.abs(tv.cpu().numpy() - v64).max()
        assert dv <= (step + 1) * 3 * 2.0 ** -24 * np.abs(v64).max()
        assert np.linalg.norm(tw.cpu().numpy() - w64) <= (step + 1) * (
            lr * scale * TOL["f32"] * np.linalg.norm(o) + 4 * 2.0 ** -24 * np.linalg.norm(w64))
        rq, rs = ref.quantize_rows(tw.cpu().numpy().reshape(b * r, c))
        assert np.array_equal(sw.cpu().numpy(), rs) and np.array_equal(wq.cpu().numpy(), ref.padded(rq))
        if wqt is not None:
            assert np.array_equal(wqt.cpu().numpy(), ref.padded(rq.T))


def test_captured():
    rng = np.random.default_rng(8)
    r, c = 140, 90
    d = dfp.make_ortho_desc(1, r, c, torch.float32)
    w0, v0 = (to_dev(matrices(rng, 1, r, c, "full")) for _ in range(2))
    g = to_dev(matrices(rng, 1, r, c, "full"))
    w, v, ws, ws2 = w0.clone(), v0.clone(), dfp.alloc_ortho_workspace(d), dfp.alloc_ortho_workspace(d)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        dfp.dfp_muon_quantize(d, 0.1, 0.9, 0.1, 1.0, w, v, g, workspace=ws)
        with torch.cuda.graph(graph, stream=side):
            dfp.dfp_muon_quantize(d, 0.1, 0.9, 0.1, 1.0, w, v, g, workspace=ws)
    torch.cuda.synchronize()
    w.copy_(w0), v.copy_(v0)
    w1, v1 = w0.clone(), v0.clone()
    for _ in range(3):
        g.copy_(to_dev(matrices(rng, 1, r, c, "full")))
        graph.replay()
        dfp.dfp_muon_quantize(d, 0.1, 0.9, 0.1, 1.0, w1, v1, g, workspace=ws2)
        torch.cuda.synchronize()
        assert torch.equal(w, w1) and torch.equal(v, v1)


def test_training_step_of_a_layer():
    """Quantise, forward, gradients, update, requantise, forward: the loop as it is used, against 64 bits."""
    rng = np.random.default_rng(21)
    m, n, k = 150, 96, 160
    x = rng.standard_normal((m, k)).astype(np.float32)
    target = rng.standard_normal((m, n)).astype(np.float32)
    w = (rng.standard_normal((n, k)) / np.sqrt(k)).astype(np.float32)
    tw, tv, tx = to_dev(w), torch.zeros(n, k, device=DEV), to_dev(x)
    ld, od = dfp.make_linear_desc(m, n, k, torch.float32), dfp.make_ortho_desc(1, n, k, torch.float32)
    ws, ows = dfp.alloc_linear_i8_workspace(ld), dfp.alloc_ortho_workspace(od)
    wq, wqt = (torch.empty(a, ref.ld(b), dtype=torch.int8, device=DEV) for a, b in ((n, k), (k, n)))
    xqt = torch.empty(k, ref.ld(m), dtype=torch.int8, device=DEV)
    sw, sx, y = torch.empty(n, device=DEV), torch.empty(m, device=DEV), torch.empty(m, n, device=DEV)
    dx, dw, db = torch.empty(m, k, device=DEV), torch.empty(n, k, device=DEV), torch.empty(n, device=DEV)
    dfp.dfp_quantize_i8(tw, wq, sw, wqt, role=dfp.ROLE_W)
    v64 = np.zeros((n, k))
    for step in range(3):
        dfp.dfp_linear_i8_fwd(ld, tx, wq, sw, y, sx=sx, xqt=xqt, workspace=ws)
        dy = (y - to_dev(target)) / m
        dfp.dfp_linear_i8_bwd_data(ld, dy, wqt, sw, dx, workspace=ws)
        dfp.dfp_linear_i8_bwd_weights(ld, dy, xqt, sx, dw, db=db, workspace=ws)
        before = tw.cpu().numpy().astype(np.float64)
        # this step from the weights and gradient outputs that the device holds
        rq, rs = ref.quantize_rows(tw.cpu().numpy())
        assert np.array_equal(wq.cpu().numpy(), ref.padded(rq)) and np.array_equal(wqt.cpu().numpy(),
                                                                                   ref.padded(rq.T))
        xq, sxr = ref.quantize_rows(x)
        yr, size = ref.product(xq, sxr, rq, rs)
        assert (np.abs(y.cpu().numpy() - yr) <= 4 * 2.0 ** -24 * size).all()
        dyh = dy.cpu().numpy().astype(np.float64)
        gq, sg = ref.quantize_rows((dyh * rs[None, :]).astype(np.float32))
        want, size = ref.product(gq, sg, rq.T)
        assert (np.abs(dx.cpu().numpy() - want) <= 4 * 2.0 ** -24 * size).all()
        gq, sg = ref.quantize_rows((dyh * sxr[:, None]).astype(np.float32).T)
        want, size = ref.product(gq, sg, xq.T)
        assert (np.abs(dw.cpu().numpy() - want) <= 4 * 2.0 ** -24 * size).all()
        dfp.dfp_muon_quantize(od, 0.02, 0.9, 0.0, 0.5, tw, tv, dw, wq, sw, wqt, workspace=ows)
        g64 = dw.cpu().numpy().astype(np.float64)
        v64 = 0.9 * v64 + g64
        o = ref.newton_schulz(g64 + 0.9 * v64, [COEF] * 5, 1e-7)
        assert np.linalg.norm(tw.cpu().numpy() - (before - 0.01 * o)) <= 0.01 * TOL["f32"] * np.linalg.norm(o) + \
            4 * 2.0 ** -24 * np.linalg.norm(before)


def test_binding_refuses():
    d = dfp.make_ortho_desc(2, 8, 16, torch.float32)
    x, ws = torch.zeros(2, 8, 16, device=DEV), dfp.alloc_ortho_workspace(d)
    with pytest.raises(ValueError):
        dfp.dfp_orthogonalize(d, x[0].contiguous(), x[0].contiguous(), workspace=ws)
    with pytest.raises(TypeError):
        dfp.dfp_orthogonalize(d, x.bfloat16(), x, workspace=ws)
    with pytest.raises(TypeError):
        dfp.dfp_muon_quantize(d, 0.1, 0.9, 0.0, 1.0, x, x.clone(), x.transpose(0, 1).contiguous().transpose(0, 1),
                              workspace=ws)
    with pytest.raises(dfp.DfpError):
        dfp.dfp_orthogonalize(d, x, x)
