"""Weight steps by orthogonalised momentum: every kernel that they take, polynomials that differ from step to step,
iterations that are taken together on the small side, and what those hold in f16 on the way.

Tolerance: six times the distance of FP32 products from 64 bits, measured here, or of 2^-22, what an operand of two
f16 numbers is off by, where FP32 comes nearer than that.  Four for operands that are off by 2^-22 where FP32 numbers
are by 2^-24, and half as much again for the products that iterations taken together add."""
import pytest
import torch

import test_gpu_tiles
from gpu_helpers import DEV, note
from paper_1802_00930_amd import dfp

pytestmark = pytest.mark.gpu


def iterate(u, steps, dtype, eps=1e-7):
    """(the orthogonalised u, the largest singular value of X before and after any step)."""
    x = u.double()
    x = x.t().contiguous() if u.shape[0] > u.shape[1] else x
    x = (x / (torch.linalg.vector_norm(x) + eps)).to(dtype)
    largest = 0.0
    for a, b, c in steps:
        g = torch.mm(x, x.t().contiguous())
        x = a * x + torch.mm(b * g + c * torch.mm(g, g), x)
        if dtype is torch.float64:
            largest = max(largest, float(torch.linalg.eigvalsh(torch.mm(x, x.t().contiguous()).cpu())[-1]) ** 0.5)
    return (x.t() if u.shape[0] > u.shape[1] else x).double(), largest


def update(dw, steps):
    """O(dw): w = 0 and lr scale = 1 leave -O(u), v = 0 and mu = 0 make u = dw."""
    b, r, c = dw.shape
    d = dfp.make_ortho_desc(b, r, c, dw.dtype, steps=len(steps), coef=steps)
    raw = torch.zeros(b * r * c + 64, device=DEV)
    raw[b * r * c:] = 7
    w, v = raw[:b * r * c].view(b, r, c), torch.zeros(b, r, c, device=DEV)
    ws = torch.full((dfp.ortho_workspace_bytes(d),), 0xff, dtype=torch.uint8, device=DEV)
    dfp.dfp_muon_quantize(d, 1.0, 0.0, 0.0, 1.0, w, v, dw, workspace=ws)
    assert torch.equal(v, dw.float()) and bool((raw[b * r * c:] == 7).all())
    return -w


def normal(seed, *shape):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device=DEV)


def assert_near(got, u, steps, times=6.0):
    want, largest = iterate(u, steps, torch.float64)
    plain, _ = iterate(u, steps, torch.float32)
    norm = torch.linalg.vector_norm(want)
    off, fp32 = (float(torch.linalg.vector_norm(y - want) / norm) for y in (got.double(), plain))
    print("off %.2e, FP32 %.2e, largest singular value %.2f" % (off, fp32, largest), flush=True)
    assert largest <= 4  # what the call is documented for
    assert off <= times * max(fp32, 2.0 ** -22), (off, fp32)  # (not so for NaN)
    return largest


# small at 0 and large away from it, alone or after one another: P_2 P_1 - q is far above q
AWAY_FROM_ZERO = {"zero": [(5.0, -20.0, 16.0), (0.0, 20.0, -20.0)],
                  "half": [(5.0, -20.0, 16.0), (0.5, 18.0, -18.0)],
                  "twice": [(5.0, -20.0, 16.0), (0.0, 20.0, -20.0), (0.25, 0.0, 0.0)] * 2}


# sizes that take iterations together, wide and tall (tests/test_mm_plan.py)
TOGETHER = [(1, 51, 8000), (1, 8000, 51)]


@pytest.mark.parametrize("name", list(AWAY_FROM_ZERO))
@pytest.mark.parametrize("b,r,c", TOGETHER + [(3, 40, 3000), (1, 100, 5000)])
def test_polynomials_that_are_large_away_from_zero(b, r, c, name):
    note("weight step %dx%dx%d %s" % (b, r, c, name))
    dw = 1e-3 * normal(r + c, b, r, c)
    got = update(dw, AWAY_FROM_ZERO[name])
    for i in range(b):
        assert_near(got[i], dw[i], AWAY_FROM_ZERO[name])


# A strong direction reaches 3.9, a singular value that the second step nearly takes to 0: a is large, and B's
# entries are as large there, far above what b and c give up to 2.
STEEP = [(3.9, 0.0, 0.0), (64.0, 0.0, -0.2766)]


def one_strong_direction(r, c):
    """Its left side on two rows, so that B's entries there are on and off the diagonal; a hundredth of it beside it."""
    left = torch.zeros(r, 1, device=DEV)
    left[0] = left[5] = 0.5 ** 0.5
    right, rest = normal(r, 1, c), normal(r + 1, r, c)
    right = right / torch.linalg.vector_norm(right)
    return 1e-3 * (left * right + 0.01 * rest / torch.linalg.matrix_norm(rest.cpu(), 2).to(DEV))


@pytest.mark.parametrize("steps", [STEEP, STEEP + [(0.3, 0.1, -0.01)]])
@pytest.mark.parametrize("r,c", [(24, 40), (24, 2000), (2000, 24), (70, 90), (51, 8000), (8000, 51)])
def test_weight_step_near_the_largest_singular_value(r, c, steps):
    note("weight step %dx%d at 3.9" % (r, c))
    dw = one_strong_direction(min(r, c), max(r, c))
    dw = (dw.t().contiguous() if r > c else dw)[None]
    assert assert_near(update(dw, steps)[0], dw[0], steps) > 3.8


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("r,c", [(24, 40), (40, 24), (70, 90)])
def test_update_near_the_largest_singular_value(r, c, t):
    """BF16: of B, whose entries sum to |B| <= 64 in squares, of A <= 16, times dB/dA <= 2 16 0.2766, and of X <= 4 a
    rounding is 2^-12: 2^-12 (64 4 + 16 8.9 4 + 64 4) = 0.27 in all; then 2^-9 of the other step and the result's
    2^-8."""
    note("update %dx%d at 3.9 %s" % (r, c, t))
    x = one_strong_direction(min(r, c), max(r, c))
    x = (x.t().contiguous() if r > c else x).to(t)[None]
    d = dfp.make_ortho_desc(1, r, c, t, steps=2, coef=STEEP)
    out = torch.empty_like(x)
    dfp.dfp_orthogonalize(d, x, out, workspace=dfp.alloc_ortho_workspace(d))
    if t is torch.float32:
        assert_near(out[0], x[0], STEEP)
        return
    want, largest = iterate(x[0], STEEP, torch.float64)
    off, norm = torch.linalg.vector_norm(out[0].double() - want), torch.linalg.vector_norm(want)
    print("off %.3f of %.1f, largest singular value %.2f" % (off, norm, largest), flush=True)
    assert 3.8 < largest <= 4 and off <= 0.27 + (2.0 ** -9 + 2.0 ** -8) * norm


# The second polynomial is steep where the first has left the singular values, some of them enlarged tenfold: taken
# together with it, what A is off by would show.
CLIFFS = [[(8.0, -24.0, 17.5), (8.0, -40.0, 50.0)], [(10.0, -25.0, 16.0), (10.0, -60.0, 60.0)],
          [(12.0, -28.0, 17.0), (12.0, -64.0, 64.0)]]


@pytest.mark.parametrize("steps", CLIFFS)
@pytest.mark.parametrize("r,c", [row[1:] for row in TOGETHER])
def test_steep_polynomials_are_not_taken_together(r, c, steps):
    note("weight step %dx%d %s" % (r, c, steps))
    rows, cols = min(r, c), max(r, c)
    dw = 1e-3 * (0.3 * normal(r, rows, cols) + normal(r + 1, rows, 1) * normal(r + 2, 1, cols))
    dw = (dw.t().contiguous() if r > c else dw)[None]
    assert_near(update(dw, steps)[0], dw[0], steps)


# The tiles of the Gram product, the polynomial (whether iterations are taken together) and the step; (2): by two
# groups of waves.  tests/test_mm_plan.py holds the names against the plans, and the lists against all that are taken.
TILES = [
    (1, 2048, 8192, "96 x 96 (2); 96 x 96 (2) together; 256 x 256"),
    (1, 8192, 2048, "96 x 96 (2); 96 x 96 (2) together; 256 x 256"),
    (1, 2050, 8190, "96 x 96 (2); 96 x 96 (2) together; 192 x 128"),
    (1, 4096, 11008, "192 x 192; 192 x 192 together; 192 x 192"),
    (1, 30, 50, "64 x 64; 64 x 64; 64 x 64"),
    (4, 641, 1385, "96 x 96 (2); 96 x 96 (2) together; 64 x 64"),
    (12, 968, 1361, "128 x 128; 128 x 128 together; 128 x 128"),
    (12, 1318, 1012, "128 x 128; 128 x 128 together; 192 x 192"),
    (16, 770, 593, "128 x 128 (2); 128 x 128 (2) together; 64 x 64"),
    (16, 1068, 852, "192 x 192; 192 x 192 together; 128 x 128"),
    (16, 1330, 1162, "256 x 256; 256 x 256 together; 128 x 128"),
    (12, 970, 1014, "128 x 128; 128 x 128; 128 x 128"),
    (16, 595, 603, "128 x 128 (2); 128 x 128 (2); 128 x 128"),
    (12, 919, 906, "192 x 192; 192 x 192; 192 x 128"),
    (16, 1169, 1198, "256 x 256; 256 x 256; 128 x 128"),
    (16, 944, 469, "128 x 128 (2); 64 x 64 together; 192 x 192"),
    (16, 467, 6514, "128 x 128, 3 slices; 64 x 64 together; 128 x 128"),
    (9, 205, 10579, "128 x 128 (2), 9 slices; 64 x 64 together; 128 x 128"),
    (2, 6736, 1420, "192 x 192, 3 slices; 128 x 128 (2) together; 128 x 128"),
    (1, 4394, 2978, "256 x 256, 3 slices; 64 x 64 together; 256 x 256"),
    (16, 1579, 65, "64 x 64, 5 slices; 64 x 64 together; 128 x 128"),
    (16, 3935, 129, "64 x 64 (2), 2 slices; 64 x 64 together; 256 x 256"),
    (3, 10984, 129, "64 x 64 (2), 14 slices; 64 x 64 together; 192 x 192"),
    (16, 666, 130, "64 x 64 (2); 64 x 64 together; 96 x 96"),
    (1, 466, 457, "64 x 64 (2); 64 x 64 (2); 64 x 64 (2)"),
]
USUAL = (3.4445, -4.7750, 2.0315)
SCHEDULES = {"usual": [USUAL] * 5,
             # to 3.8, near the largest that the units are for, and back to 1.5
             "reach": [USUAL] * 3 + [(3.2, 0.0, 0.0), (0.6, -0.03, 0.001)]}


@pytest.mark.parametrize("name", list(SCHEDULES))
@pytest.mark.parametrize("b,r,c,tiles", TILES)
def test_tiles(b, r, c, tiles, name):
    """Strong directions above weaker ones.  An error of A, 2^-22, grows by 140 and by the slope 8.9 of the polynomial
    that it enters, 3e-4 at most; "reach" takes every direction times 1.2 to 1.9 in the end, which adds to that as much
    again relative to its norm at most."""
    note("weight step %dx%dx%d %s %s" % (b, r, c, name, tiles))
    k = max(1, min(r, c) // 16)
    dw = 1e-3 * (0.3 * normal(r + 3 * c, b, r, c) + torch.matmul(normal(r, b, r, k), normal(c, b, k, c)) / k ** 0.5)
    got = update(dw, SCHEDULES[name])
    worst = 0.0
    for i in range(b):
        x = dw[i].double()
        x = x.t().contiguous() if r > c else x
        x = x / (torch.linalg.vector_norm(x) + 1e-7)
        for ca, cb, cc in SCHEDULES[name]:
            a = torch.mm(x, x.t().contiguous())
            x = ca * x + torch.mm(cb * a + cc * torch.mm(a, a), x)
        x = x.t() if r > c else x
        off = float(torch.linalg.vector_norm(got[i].double() - x) / torch.linalg.vector_norm(x))
        worst = max(worst, off)
        assert off <= (3e-4 if name == "usual" else 6e-4), (i, off)
    print("off %.2e" % worst, flush=True)


@pytest.mark.parametrize("b,r,c", [(3, 400, 420), (3, 100, 9000), (3, 9000, 100)])
def test_a_matrix_out_of_range_leaves_the_others(b, r, c):
    """The middle matrix is one direction, which the first step takes to 30, far beyond 4; the others' stay at 3."""
    note("weight step %dx%dx%d, one out of range" % (b, r, c))
    steps = [(30.0, 0.0, 0.0), (0.1, 0.0, 0.0)]
    dw = 1e-3 * normal(r, b, r, c)
    dw[1] = 1e-3 * normal(r + 1, r, 1) * normal(r + 2, 1, c)
    got = update(dw, steps)
    for i in (0, 2):
        assert_near(got[i], dw[i], steps)


# products and updates on the kernels that the lists of test_gpu_tiles.py leave out
PRODUCTS = [(1033, 1, 68773), (1153, 302, 33238)]  # 96 x 96 by two groups, in slices
UPDATES = [("bf16", 16, 581, 604)]                 # Gram product on whole 128 x 128 tiles


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, t):
    test_gpu_tiles.test_product(m, n, k, t)


@pytest.mark.parametrize("t,b,r,c", UPDATES)
def test_orthogonalize(t, b, r, c):
    test_gpu_tiles.test_orthogonalize(t, b, r, c)


@pytest.mark.parametrize("weak", [0.1, 0.01, 0.001])
@pytest.mark.parametrize("r,c,k", [(256, 256, 32), (512, 512, 1), (300, 700, 18), (700, 300, 1)])
def test_bf16_update_of_strong_directions_above_weak_ones(r, c, k, weak):
    """Documented for the usual coefficients: what single f16 numbers add stays below half of BF16's half step, 2^-9,
    and the result's own rounding adds at most 2^-8 / sqrt(3)."""
    note("update %dx%d rank %d, %g beside it" % (r, c, k, weak))
    x = weak * normal(r, r, c) * torch.exp(0.5 * normal(c, r, 1)) + normal(1, r, k) @ normal(2, k, c) / k ** 0.5
    x = x.bfloat16()
    d = dfp.make_ortho_desc(1, r, c, torch.bfloat16)
    out = torch.empty_like(x)
    dfp.dfp_orthogonalize(d, x, out, workspace=dfp.alloc_ortho_workspace(d))
    want, _ = iterate(x, SCHEDULES["usual"], torch.float64)
    off = float(torch.linalg.vector_norm(out.double() - want) / torch.linalg.vector_norm(want))
    print("off %.2e" % off, flush=True)
    assert off <= (2.0 ** -18 + 2.0 ** -16 / 3) ** 0.5


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("b,r,c", [(12, 512, 512), (1, 1000, 333), (1, 51, 8000), (2, 1469, 7439)])
def test_calls_repeat_themselves(b, r, c, t):
    """Bit for bit, whatever the workspace holds and whatever runs beside them."""
    note("update %dx%dx%d %s twice" % (b, r, c, t))
    x = normal(r, b, r, c).to(t)
    d = dfp.make_ortho_desc(b, r, c, t)
    n = dfp.ortho_workspace_bytes(d)
    streams = [torch.cuda.Stream() for _ in range(2)]
    ws = [torch.full((n,), g, dtype=torch.uint8, device=DEV) for g in (0xff, 0)]
    outs = [torch.empty_like(x) for _ in range(2)]
    w = [normal(1, b, r, c) for _ in range(2)]
    v = [normal(2, b, r, c) for _ in range(2)]
    torch.cuda.synchronize()
    for i, s in enumerate(streams):
        dfp.dfp_orthogonalize(d, x, outs[i], workspace=ws[i], stream=s)
        dfp.dfp_muon_quantize(d, 0.02, 0.95, 0.1, 0.2, w[i], v[i], x, workspace=ws[i], stream=s)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(w[0], w[1]) and torch.equal(v[0], v[1])
