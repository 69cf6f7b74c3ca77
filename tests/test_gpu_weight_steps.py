"""Weight steps by orthogonalised momentum whose polynomials differ from step to step: ones that take iterations
together on the small side, and what they hold in f16 on the way.

Tolerance: six times the distance of FP32 products from 64 bits, measured here, or of 2^-22, what an operand of two
f16 numbers is off by, where FP32 comes nearer than that.  Four for operands that are off by 2^-22 where FP32 numbers
are by 2^-24, and half as much again for the products that iterations taken together add."""
import pytest
import torch

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


@pytest.mark.parametrize("name", list(AWAY_FROM_ZERO))
@pytest.mark.parametrize("b,r,c", [(1, 51, 8000), (1, 8000, 51), (3, 40, 3000), (1, 100, 5000)])
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
@pytest.mark.parametrize("r,c", [(24, 40), (24, 2000), (2000, 24), (70, 90)])
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
@pytest.mark.parametrize("r,c", [(51, 8000), (8000, 51)])
def test_steep_polynomials_are_not_taken_together(r, c, steps):
    note("weight step %dx%d %s" % (r, c, steps))
    rows, cols = min(r, c), max(r, c)
    dw = 1e-3 * (0.3 * normal(r, rows, cols) + normal(r + 1, rows, 1) * normal(r + 2, 1, cols))
    dw = (dw.t().contiguous() if r > c else dw)[None]
    assert_near(update(dw, steps)[0], dw[0], steps)
