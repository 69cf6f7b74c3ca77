"""Every tile and way of slicing that the products' estimates choose, at sizes that
reach each of them, against 64-bit products on the GPU (integers are exact there).
Tolerances as in test_gpu_linear_i8.py and test_gpu_ortho.py."""
import numpy as np
import pytest
import torch

import linear_ref as ref
from gpu_helpers import DEV, note
from paper_1802_00930_amd import dfp

pytestmark = pytest.mark.gpu

# m, n, k: the tile that the estimate chooses, and slices of the reduction
PRODUCTS = [
    (66, 16892, 100),       # 96 x 96
    (1500, 1500, 500),      # 96 x 96
    (134, 32975, 200),      # 192 x 192
    (3000, 3000, 257),      # 192 x 192
    (49252, 135, 40),       # 96 x 96
    (4000, 4090, 300),      # 256 x 256
    (33709, 70, 129),       # 192 x 128
    (3000, 2000, 1000),     # 192 x 128
    (68, 26785, 300),       # 128 x 128
    (2000, 2000, 200),      # 128 x 128
    (1100, 1500, 700),      # 64 x 64
    (65, 3, 1965),          # 64 x 64, 16 slices
    (200, 300, 30000),      # 64 x 64 by two groups, 8 slices
    (69, 2051, 3667),       # 64 x 64 by two groups
    (73, 6667, 6926),       # 64 x 64 by two groups
    (3258, 67, 15308),      # 64 x 64 by two groups, 2 slices
    (3248, 148, 22892),     # 128 x 128 by two groups, 4 slices
    (3597, 148, 75337),     # 192 x 192, 8 slices
    (64, 1, 1),             # 64 x 64
    (40, 9000, 3000),       # 64 x 64 by two groups
    (24, 5000, 8192),       # 64 x 64 by two groups, 2 slices
    (16720, 17, 3113),      # 96 x 96 by two groups
    (1091, 20, 63062),      # 64 x 64 by two groups, 8 slices
    (71, 2105, 8158),       # 96 x 96, 8 slices
    (195, 2123, 62434),     # 256 x 256, 16 slices
    (1085, 195, 26458),     # 192 x 128, 16 slices
    (1077, 102, 50733),     # 128 x 128 by two groups, 16 slices
    (16503, 97, 1641),      # 128 x 128 by two groups
    (3151, 130, 26571),     # 192 x 192, 8 slices
    (99, 4387, 91434),      # 128 x 128, 16 slices
    (1914, 33, 2132),       # 64 x 64 by two groups
    (64, 35919, 18),        # rows of a batch
    (63124, 130, 40),       # 256 x 256
]


@pytest.mark.parametrize("t", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k, t):
    note("tiles %dx%dx%d %s" % (m, n, k, t))
    g = torch.Generator(device=DEV)
    g.manual_seed(m + n + k)
    a, b = (torch.zeros(r, ref.ld(k), dtype=torch.int8, device=DEV) for r in (m, n))
    for x in (a, b):
        x[:, :k] = torch.randint(-127, 128, (x.shape[0], k), generator=g, device=DEV, dtype=torch.int8)
    sa, sb = (torch.rand(r, generator=g, device=DEV) * 2.0 ** -6 for r in (m, n))
    bias = torch.randn(n, generator=g, device=DEV)
    d = dfp.make_linear_desc(m, n, k, t)
    raw = torch.full((m * n + 256,), 77, dtype=t, device=DEV)
    ws = torch.full((dfp.linear_i8_workspace_bytes(d),), 0x81, dtype=torch.uint8, device=DEV)
    out = raw[:m * n].view(m, n)
    dfp.dfp_gemm_i8(d, a, sa, b, sb, out, bias=bias, workspace=ws)
    y = torch.mm(a.double(), b.double().t()) * sa.double()[:, None] * sb.double()[None, :]
    size = y.abs() + bias.double().abs()[None, :]
    y = y + bias.double()[None, :]
    half = 2.0 ** -24 if t is torch.float32 else 2.0 ** -8
    tol = 4 * 2.0 ** -24 * (size + y.abs()) + half * 1.0001 * y.abs()
    assert bool(((out.double() - y).abs() <= tol).all())
    assert bool((raw[m * n:] == 77).all())


# the tiles of the Gram product, the polynomial and the step, (2) by two groups of waves;
# operands of one f16 number (BF16) or two
ORTHO = [
    ("bf16", 9, 1175, 924),    # 96 x 96; 96 x 96; 192 x 128
    ("bf16", 1, 2641, 1146),   # 64 x 64 (2); 64 x 64 (2); 64 x 64
    ("bf16", 9, 875, 977),     # 128 x 128 (2); 128 x 128; 128 x 128
    ("bf16", 1, 7154, 1009),   # 96 x 96 (2), 3 slices; 64 x 64; 192 x 192
    ("bf16", 9, 1154, 1109),   # 192 x 192; 192 x 192; 256 x 256
    ("bf16", 1, 1312, 14953),  # 96 x 96 (2), 2 slices; 64 x 64 (2); 192 x 128
    ("bf16", 9, 1550, 1928),   # 256 x 256; 256 x 256; 256 x 256
    ("bf16", 4, 996, 10316),   # 192 x 192, 3 slices; 64 x 64; 256 x 256
    ("bf16", 9, 134, 1234),    # 64 x 64 (2); 64 x 64; 96 x 96
    ("bf16", 9, 3896, 67),     # 64 x 64, 9 slices; 64 x 64; 192 x 128
    ("bf16", 4, 131, 8562),    # 64 x 64, 10 slices; 64 x 64; 96 x 96
    ("bf16", 9, 6071, 144),    # 64 x 64 (2), 4 slices; 64 x 64; 96 x 96
    ("f32", 9, 1038, 917),     # 96 x 96 (2); 96 x 96 (2); 64 x 64
    ("f32", 4, 531, 1469),     # 64 x 64 (2); 64 x 64 (2); 128 x 128 (2)
    ("f32", 9, 819, 921),      # 128 x 128 (2); 128 x 128 (2); 192 x 192
    ("f32", 1, 849, 4228),     # 64 x 64 (2), 2 slices; 64 x 64 (2); 128 x 128 (2)
    ("f32", 9, 1807, 1303),    # 192 x 192; 192 x 192; 192 x 128
    ("f32", 1, 9751, 1286),    # 96 x 96 (2), 2 slices; 64 x 64 (2); 256 x 256
    ("f32", 9, 1693, 1632),    # 256 x 256; 256 x 256; 192 x 192
    ("f32", 1, 1995, 7899),    # 96 x 96 (2); 96 x 96 (2); 256 x 256
    ("f32", 1, 11162, 130),    # 64 x 64, 32 slices; 64 x 64; 96 x 96
    ("f32", 9, 69, 3646),      # 64 x 64, 9 slices; 64 x 64; 64 x 64
    ("f32", 4, 10127, 129),    # 64 x 64 (2), 10 slices; 64 x 64; 192 x 192
    ("f32", 4, 140, 15184),    # 64 x 64 (2), 10 slices; 64 x 64; 192 x 128
    ("bf16", 9, 11475, 976),   # 128 x 128, 3 slices; 64 x 64; 192 x 128
    ("bf16", 2, 987, 6115),    # 128 x 128 (2), 3 slices; 96 x 96; 128 x 128
    ("bf16", 2, 1469, 7439),   # 192 x 192, 3 slices; 128 x 128 (2); 192 x 128
    ("bf16", 1, 8977, 2972),   # 256 x 256, 3 slices; 192 x 192; 192 x 192
    ("bf16", 4, 680, 800),     # 96 x 96; 64 x 64; 64 x 64
    ("bf16", 4, 646, 1917),    # 96 x 96 (2); 64 x 64; 192 x 128
    ("bf16", 2, 8356, 513),    # 96 x 96 (2), 6 slices; 64 x 64; 192 x 128
    ("bf16", 2, 1563, 1538),   # 128 x 128 (2); 128 x 128 (2); 192 x 128
    ("bf16", 1, 1043, 1123),   # 64 x 64 (2); 64 x 64 (2); 96 x 96
    ("bf16", 1, 1873, 1604),   # 96 x 96 (2); 96 x 96 (2); 128 x 128 (2)
    ("bf16", 9, 2850, 65),     # 64 x 64, 9 slices; 64 x 64; 128 x 128
    ("bf16", 1, 4121, 709),    # 64 x 64 (2), 3 slices; 64 x 64; 128 x 128 (2)
    ("bf16", 4, 77, 10474),    # 64 x 64, 21 slices; 64 x 64; 192 x 192
    ("bf16", 9, 6971, 152),    # 64 x 64 (2), 4 slices; 64 x 64; 256 x 256
    ("bf16", 1, 926, 899),     # 64 x 64; 64 x 64; 64 x 64 (2)
    ("bf16", 1, 1420, 1293),   # 64 x 64 (2); 64 x 64 (2); 96 x 96 (2)
    ("bf16", 9, 1309, 650),    # 128 x 128 (2); 64 x 64; 192 x 192
    ("f32", 9, 1200, 1250),    # 128 x 128; 128 x 128; 256 x 256
    ("f32", 4, 7483, 1010),    # 128 x 128, 3 slices; 128 x 128 (2); 192 x 128
    ("f32", 9, 1120, 650),     # 128 x 128 (2); 64 x 64; 192 x 192
    ("f32", 9, 193, 11889),    # 128 x 128 (2), 9 slices; 64 x 64; 128 x 128
    ("f32", 2, 1445, 7276),    # 192 x 192, 3 slices; 128 x 128 (2); 192 x 128
    ("f32", 1, 3035, 4387),    # 256 x 256, 3 slices; 64 x 64; 256 x 256
    ("f32", 1, 15394, 3),      # 64 x 64 (2), 31 slices; 64 x 64; 64 x 64
    ("f32", 4, 654, 665),      # 96 x 96 (2); 96 x 96 (2); 64 x 64
    ("f32", 9, 13104, 130),    # 96 x 96 (2), 9 slices; 64 x 64; 192 x 192
    ("f32", 4, 1009, 1078),    # 128 x 128 (2); 128 x 128 (2); 192 x 128
    ("f32", 1, 479, 487),      # 64 x 64 (2); 64 x 64 (2); 64 x 64 (2)
    ("f32", 2, 66, 12289),     # 64 x 64, 30 slices; 64 x 64; 128 x 128
    ("f32", 2, 461, 3194),     # 64 x 64 (2), 3 slices; 64 x 64 (2); 128 x 128 (2)
    ("f32", 4, 8426, 133),     # 64 x 64 (2), 10 slices; 64 x 64; 192 x 192
    ("f32", 4, 15888, 157),    # 64 x 64 (2), 10 slices; 64 x 64; 256 x 256
    ("f32", 1, 653, 1650),     # 64 x 64 (2), 3 slices; 64 x 64 (2); 96 x 96 (2)
]
COEF = (3.4445, -4.7750, 2.0315)


@pytest.mark.parametrize("t,b,r,c", ORTHO)
def test_orthogonalize(t, b, r, c):
    note("ortho tiles %s %dx%dx%d" % (t, b, r, c))
    dt = torch.float32 if t == "f32" else torch.bfloat16
    g = torch.Generator(device=DEV)
    g.manual_seed(r + c)
    x = (torch.randn(b, r, c, generator=g, device=DEV) * torch.exp(0.5 * torch.randn(b, r, 1, generator=g, device=DEV)))
    x = (1e-3 * x).to(dt)
    d = dfp.make_ortho_desc(b, r, c, dt)
    raw = torch.full((b * r * c + 256,), 7, dtype=dt, device=DEV)
    out = raw[:b * r * c].view(b, r, c)
    ws = torch.full((dfp.ortho_workspace_bytes(d),), 0xff, dtype=torch.uint8, device=DEV)
    dfp.dfp_orthogonalize(d, x, out, workspace=ws)
    for i in range(b):
        u = x[i].double()
        u = u.t().contiguous() if r > c else u
        u = u / (torch.linalg.vector_norm(u) + 1e-7)
        for _ in range(5):
            a = torch.mm(u, u.t().contiguous())
            u = COEF[0] * u + torch.mm(COEF[1] * a + COEF[2] * torch.mm(a, a), u)
        u = u.t() if r > c else u
        off = float(torch.linalg.vector_norm(out[i].double() - u) / torch.linalg.vector_norm(u))
        assert np.isfinite(off) and off <= (2e-4 if t == "f32" else 3e-3), (i, off)
    assert bool((raw[b * r * c:] == 7).all())


# weight steps that iterate on the small side, wide and tall, a batch, and beside them ones that do not
MUON = [(1, 1024, 4096), (1, 4096, 1024), (1, 2200, 1000), (3, 200, 2000), (1, 20000, 200), (2, 130, 9000),
        (1, 64, 8000), (1, 512, 2048), (1, 1500, 1500)]
SCHEDULES = {
    "same": [COEF] * 5,
    "one": [COEF],
    "two": [COEF] * 2,
    "eight": [(2.0, -1.5, 0.5)] * 8,
    # coefficients of their own for each step, the first far above the others: within [0, 2] on [0, 1]
    "falling": [(8.287, -23.596, 17.300), (4.107, -2.948, 0.545), (3.949, -2.909, 0.552), (3.318, -2.488, 0.510),
                (2.301, -1.669, 0.419)],
    # the middle of [0, 1] grows most
    "middle": [(1.2, 0.3, -0.5)] * 8,
    # "falling" rounded further: from 1 they end above 1000, past the documented range (4)
    "out of range": [(8.2, -23.0, 17.0), (4.1, -2.9, 0.55), (3.9, -2.8, 0.55), (3.3, -2.4, 0.5), (2.0, -1.5, 0.5)],
}


@pytest.mark.parametrize("kind", ["full", "low_rank"])
@pytest.mark.parametrize("coef", list(SCHEDULES))
@pytest.mark.parametrize("b,r,c", MUON)
def test_muon(b, r, c, coef, kind):
    """The update's tolerance is that of single iterations, twice: an error of A grows by
    (a a')^2 = 140 at most before X is looked at again, of A's 2^-22: 3.4e-5, six of which
    (B has |b| + 2 |c| of it) stay under 2e-4."""
    note("muon tiles %dx%dx%d %s %s" % (b, r, c, coef, kind))
    steps = SCHEDULES[coef]
    g = torch.Generator(device=DEV)
    g.manual_seed(r * 3 + c)
    normal = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    u = normal(b, r, c) * torch.exp(0.5 * normal(b, r, 1))
    if kind == "low_rank":
        k = min(r, c) // 16
        u = 0.3 * u + torch.stack([normal(r, k) @ normal(k, c) for _ in range(b)])
    dw = (1e-3 * u).contiguous()
    d = dfp.make_ortho_desc(b, r, c, torch.float32, steps=len(steps), coef=steps)
    # w = 0 and lr scale = 1 leave -O(u), v = 0 and mu = 0 make u = dw
    w, v = torch.zeros(b, r, c, device=DEV), torch.zeros(b, r, c, device=DEV)
    ws = torch.full((dfp.ortho_workspace_bytes(d),), 0xff, dtype=torch.uint8, device=DEV)
    dfp.dfp_muon_quantize(d, 1.0, 0.0, 0.0, 1.0, w, v, dw, workspace=ws)
    assert torch.equal(v, dw)
    for i in range(b):
        x = dw[i].double()
        x = x.t().contiguous() if r > c else x
        x = x / (torch.linalg.vector_norm(x) + 1e-7)
        largest = 0.0
        for ca, cb, cc in d.coef[:len(steps)]:
            a = torch.mm(x, x.t().contiguous())
            x = ca * x + torch.mm(cb * a + cc * torch.mm(a, a), x)
            z = torch.ones(x.shape[0], 1, dtype=torch.float64, device=DEV)
            for _ in range(20):  # the largest singular value, from below
                z = torch.mm(x, torch.mm(x.t().contiguous(), z / torch.linalg.vector_norm(z)))
            largest = max(largest, float(torch.linalg.vector_norm(z)) ** 0.5)
        if largest > 4:
            assert coef == "out of range"
            continue
        x = x.t() if r > c else x
        off = float(torch.linalg.vector_norm(w[i].double() + x) / torch.linalg.vector_norm(x))
        print("off %.2e, largest %.2f" % (off, largest))
        assert np.isfinite(off) and off <= 4e-4, off
