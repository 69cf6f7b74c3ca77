"""Operators of INT8 linear layers and of the orthogonalised weight update.

Kinds of case:

* ``fwd``    y = x W^T + bias with tokens quantised to INT8 on the way in and
  weights held as INT8 with a scale per output channel;
* ``gemm``   the INT8 product alone, of operands that are quantised already;
* ``bwd``    backward-data and backward-weights of that layer;
* ``train``  forward and both gradients;
* ``quant``  rows of a matrix to INT8, one scale each;
* ``ortho``  matrices orthogonalised by Newton-Schulz products;
* ``muon``   the weight step that orthogonalises the momentum.

INT8 operands are [rows][ld] with ld = cols rounded up to 128 and zeros in the
padding.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
COEF = (3.4445, -4.7750, 2.0315)
STEPS, EPS = 5, 1e-7
LR, MU, WD, SCALE = 0.02, 0.95, 0.1, 0.2
LARGEST = 2 * 16384 * 8192 * 8192


def _linear(name, kind, m, n, k, t, bias=True):
    return {"name": name, "kind": kind, "m": m, "n": n, "k": k, "type": t, "bias": bias}


def _matrix(name, kind, batch, rows, cols, t):
    return {"name": name, "kind": kind, "batch": batch, "rows": rows, "cols": cols, "type": t}


def listed():
    return [
        # a single token in serving: the weights' bytes and the launch are all there is
        _linear("fwd_token", "fwd", 1, 4096, 4096, "bf16"),
        # a batch of sequences that each decode one token
        _linear("fwd_batch", "fwd", 24, 8192, 2048, "bf16", bias=False),
        # a prompt
        _linear("fwd_prompt", "fwd", 4096, 4096, 4096, "bf16"),
        # no size a multiple of any tile
        _linear("fwd_ragged", "fwd", 777, 1003, 1111, "f32"),
        # many prompts through a wide layer: the largest
        _linear("fwd_large", "fwd", 16384, 8192, 8192, "bf16", bias=False),
        # the benchmark's fully connected layer on operands that are INT8 already
        _linear("gemm_fc", "gemm", 64, 1000, 2048, "f32"),
        # gradients of an odd layer in half precision
        _linear("bwd_odd", "bwd", 1500, 1000, 2051, "f16"),
        # one layer of a training step
        _linear("train_layer", "train", 8192, 2048, 2048, "bf16"),
        # weights to INT8 after a step
        _matrix("quant_weights", "quant", 1, 8192, 2048, "f32"),
        # the attention matrices of several small layers at once
        _matrix("ortho_layers", "ortho", 12, 512, 512, "bf16"),
        # a tall matrix of odd sizes, in FP32
        _matrix("ortho_tall", "ortho", 1, 1000, 333, "f32"),
        # the update of a wide layer's FP32 master weights
        _matrix("muon_wide", "muon", 1, 2048, 8192, "f32"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["fwd", "fwd", "gemm", "bwd", "train", "quant", "ortho", "muon"])
    if kind in ("fwd", "gemm", "bwd", "train"):
        m = _log(rng, 1, 16384)
        n, k = _log(rng, 64, 8192), _log(rng, 64, 8192)
        if kind == "train":
            m, n, k = min(m, 8192), min(n, 4096), min(k, 4096)
        return {"kind": kind, "m": m, "n": n, "k": k, "type": rng.choice(["bf16", "bf16", "f16", "f32"]),
                "bias": rng.random() < 0.5}
    t = rng.choice(["f32", "bf16"])
    if kind == "quant":
        return {"kind": kind, "batch": 1, "rows": _log(rng, 1, 8192), "cols": _log(rng, 64, 8192), "type": t}
    rows, cols = _log(rng, 64, 4096), _log(rng, 64, 4096)
    if rng.random() < 0.4:  # sides of tiles too, as most weights have
        rows, cols = -(-rows // 64) * 64, -(-cols // 64) * 64
    batch = _log(rng, 1, 16) if kind == "ortho" else 1
    while batch > 1 and batch * _ortho_flops(rows, cols) > LARGEST / 8:
        batch //= 2
    return {"kind": kind, "batch": batch, "rows": rows, "cols": cols, "type": t}


def _ld(cols):
    return -(-cols // 128) * 128


def _ortho_flops(rows, cols):
    r, c = min(rows, cols), max(rows, cols)
    return STEPS * (3 * r * r * c + r * r * r)  # the two symmetric products count half


def work(case):
    if case["kind"] in ("quant", "ortho", "muon"):
        n = case["batch"] * case["rows"] * case["cols"]
        e = 4 if case["type"] == "f32" else 2
        if case["kind"] == "quant":
            return {"bytes": n * (e + 1) + 4 * case["rows"], "flops": 2 * n}
        flops = case["batch"] * _ortho_flops(case["rows"], case["cols"])
        return {"bytes": n * (2 * e if case["kind"] == "ortho" else 16 + e), "flops": flops}
    m, n, k = case["m"], case["n"], case["k"]
    e = 4 if case["type"] == "f32" else 2
    one = 2 * m * n * k
    x, y = e * m * k, e * m * n
    grads = y + n * k + x + 4 * n * k + 4 * n  # dy and the weights; dx, dw and db
    return {"fwd": {"bytes": x + n * k + y + 8 * n, "flops": one},
            "gemm": {"bytes": m * k + n * k + y + 4 * m + 8 * n, "flops": one},
            "bwd": {"bytes": grads + m * k, "flops": 2 * one},
            "train": {"bytes": x + n * k + y + 8 * n + grads, "flops": 3 * one}}[case["kind"]]


# ------------------------------------------------------------------ inputs

def _pad(q):
    """INT8 [rows][cols] in the operands' layout."""
    out = torch.zeros(q.shape[0], _ld(q.shape[1]), dtype=torch.int8, device=q.device)
    out[:, :q.shape[1]] = q
    return out


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    t = TYPES[case["type"]]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    s = dict(case)
    if case["kind"] in ("quant", "ortho", "muon"):
        b, r, c = case["batch"], case["rows"], case["cols"]
        if case["kind"] == "quant":
            s["src"] = (normal(r, c) * (0.02 * torch.exp(normal(r, 1)))).to(t)
            return s
        # gradients: a few strong directions above noise whose rows differ in size
        rank = max(1, min(r, c) // 16)
        u = 0.3 * normal(b, r, c) * torch.exp(0.5 * normal(b, r, 1)) + torch.matmul(normal(b, r, rank), normal(b, rank, c)) / math.sqrt(rank)
        if case["kind"] == "ortho":
            s["x"] = (1e-3 * u).to(t)
            return s
        s["dw"] = (1e-3 * u[0]).to(t)
        s["v"] = 1e-3 * normal(r, c)
        s["w"] = normal(r, c) / math.sqrt(c)
        return s
    m, n, k = case["m"], case["n"], case["k"]
    # weights as the program keeps them: INT8, both layouts, a scale for each output channel
    w = normal(n, k) * math.sqrt(2.0 / k)
    amax = w.abs().amax(1)
    s["sw"] = amax / 127
    wq = torch.round(w / s["sw"][:, None]).clamp_(-127, 127).to(torch.int8)
    s["wq"], s["wqt"] = _pad(wq), _pad(wq.t())
    s["b"] = 0.1 * normal(n) if case["bias"] else None
    # activations: some channels far larger than the rest
    x = normal(m, k) * torch.exp(0.5 * normal(k))
    if case["kind"] == "gemm":
        s["sx"] = x.abs().amax(1) / 127
        s["xq"] = _pad(torch.round(x / s["sx"][:, None]).clamp_(-127, 127).to(torch.int8))
        return s
    if case["kind"] != "bwd":
        s["x"] = x.to(t)
    else:  # what the forward call left for the backward ones
        s["sx"] = x.abs().amax(1) / 127
        s["xqt"] = _pad(torch.round(x / s["sx"][:, None]).clamp_(-127, 127).to(torch.int8).t())
    if case["kind"] in ("bwd", "train"):
        # gradients: tokens of very different weight (scaled up as losses in half precision are)
        s["dy"] = (normal(m, n) * torch.exp(normal(m, 1))).to(t)
    return s


# -------------------------------------------------------------- plain forms

def _rows_to_i8(x):
    """(integers as FP32, scales) of the rows of an FP32 matrix."""
    s = (x.abs().amax(1).double() / 127).float()
    q = torch.round(x.double() / s.double()[:, None]).clamp_(-127, 127)
    return torch.where(s[:, None] > 0, q, torch.zeros_like(q)).float(), s


def _plain_fwd(xq, sx, wq, sw, b, t):
    y = torch.matmul(xq, wq.float().t()) * sx[:, None] * sw[None, :]
    return (y if b is None else y + b[None, :]).to(t)


def _plain_bwd(s, xqt, sx):
    m, n, k, t = s["m"], s["n"], s["k"], TYPES[s["type"]]
    dy = s["dy"].float()
    gq, sg = _rows_to_i8(dy * s["sw"][None, :])
    dx = (torch.matmul(gq, s["wqt"][:, :n].float().t()) * sg[:, None]).to(t)
    gq, sg = _rows_to_i8((dy * sx[:, None]).t())
    dw = torch.matmul(gq, xqt.t()) * sg[:, None]
    return {"dx": dx, "dw": dw, "db": dy.sum(0)}


def _plain_ortho(u):
    """u FP32 [batch][rows][cols]."""
    flip = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if flip else u
    norm = torch.sqrt(x.double().square().sum((1, 2), keepdim=True))
    x = (x.double() / (norm + EPS)).float()
    a, b, c = COEF
    for _ in range(STEPS):
        aa = torch.matmul(x, x.transpose(1, 2))
        aa = b * aa + c * torch.matmul(aa, aa)
        x = a * x + torch.matmul(aa, x)
    return x.transpose(1, 2).contiguous() if flip else x


def _plain(s):
    kind, t = s["kind"], TYPES[s["type"]]
    if kind == "quant":
        q, sc = _rows_to_i8(s["src"].float())
        return {"values": q * sc[:, None], "scale": sc}
    if kind == "ortho":
        return _plain_ortho(s["x"].float()).to(t)
    if kind == "muon":
        g = s["dw"].float()
        s["v"].mul_(MU).add_(g)
        o = _plain_ortho((g + MU * s["v"])[None])[0]
        s["w"].mul_(1 - LR * WD).sub_(LR * SCALE * o)
        return {"w": s["w"], "v": s["v"]}
    k = s["k"]
    if kind == "gemm":
        return _plain_fwd(s["xq"][:, :k].float(), s["sx"], s["wq"][:, :k], s["sw"], s["b"], t)
    if kind == "bwd":
        return _plain_bwd(s, s["xqt"][:, :s["m"]].float(), s["sx"])
    xq, sx = _rows_to_i8(s["x"].float())
    y = _plain_fwd(xq, sx, s["wq"][:, :k], s["sw"], s["b"], t)
    if kind == "fwd":
        return y
    return {"y": y, **_plain_bwd(s, xq.t(), sx)}


# --------------------------------------------------------- the framework's calls

def _plan(s):
    """Descriptor, workspace and output buffers, made at a state's first pass and kept by the program."""
    from paper_1802_00930_amd import dfp
    kind, t = s["kind"], TYPES[s["type"]]
    p = {"dfp": dfp}

    def new(*shape, dtype):
        return torch.empty(*shape, dtype=dtype, device=DEV)

    if kind == "quant":
        p["q"] = new(s["rows"], dfp.i8_ld(s["cols"]), dtype=torch.int8)
        p["scale"] = new(s["rows"], dtype=torch.float32)
        return p
    if kind in ("ortho", "muon"):
        p["d"] = dfp.make_ortho_desc(s["batch"], s["rows"], s["cols"], t, steps=STEPS, eps=EPS, coef=COEF)
        p["ws"] = dfp.alloc_ortho_workspace(p["d"], DEV)
        if kind == "ortho":
            p["out"] = torch.empty_like(s["x"])
        return p
    m, n, k = s["m"], s["n"], s["k"]
    p["d"] = dfp.make_linear_desc(m, n, k, t)
    p["ws"] = dfp.alloc_linear_i8_workspace(p["d"], DEV)
    if kind != "bwd":
        p["y"] = new(m, n, dtype=t)
    if kind == "train":
        p["sx"] = new(m, dtype=torch.float32)
        p["xqt"] = new(k, dfp.i8_ld(m), dtype=torch.int8)
    if kind in ("bwd", "train"):
        p["dx"], p["dw"], p["db"] = new(m, k, dtype=t), new(n, k, dtype=torch.float32), new(n, dtype=torch.float32)
    return p


def _own(s):
    p = s.get("plan")
    if p is None:
        p = s["plan"] = _plan(s)
    dfp, kind = p["dfp"], s["kind"]
    if kind == "quant":
        dfp.dfp_quantize_i8(s["src"], p["q"], p["scale"])
        return {"values": p["q"][:, :s["cols"]] * p["scale"][:, None], "scale": p["scale"]}
    if kind == "ortho":
        dfp.dfp_orthogonalize(p["d"], s["x"], p["out"], workspace=p["ws"])
        return p["out"]
    if kind == "muon":
        dfp.dfp_muon_quantize(p["d"], LR, MU, WD, SCALE, s["w"], s["v"], s["dw"], nesterov=True, workspace=p["ws"])
        return {"w": s["w"], "v": s["v"]}
    if kind == "gemm":
        dfp.dfp_gemm_i8(p["d"], s["xq"], s["sx"], s["wq"], s["sw"], p["y"], bias=s["b"], workspace=p["ws"])
        return p["y"]
    if kind == "fwd":
        dfp.dfp_linear_i8_fwd(p["d"], s["x"], s["wq"], s["sw"], p["y"], bias=s["b"], workspace=p["ws"])
        return p["y"]
    xqt, sx = s.get("xqt"), s.get("sx")
    if kind == "train":
        xqt, sx = p["xqt"], p["sx"]
        dfp.dfp_linear_i8_fwd(p["d"], s["x"], s["wq"], s["sw"], p["y"], bias=s["b"], sx=sx, xqt=xqt, workspace=p["ws"])
    dfp.dfp_linear_i8_bwd_data(p["d"], s["dy"], s["wqt"], s["sw"], p["dx"], workspace=p["ws"])
    dfp.dfp_linear_i8_bwd_weights(p["d"], s["dy"], xqt, sx, p["dw"], db=p["db"], workspace=p["ws"])
    grads = {"dx": p["dx"], "dw": p["dw"], "db": p["db"]}
    return {"y": p["y"], **grads} if kind == "train" else grads


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------ 64 bits

def _scaled(x):
    """x FP64 [rows][cols]: (integers, scales). The scale is the FP32 number that a caller gets."""
    s = torch.amax(torch.abs(x), dim=1, keepdim=True).div(127.0).float().double()
    q = torch.where(s == 0, torch.zeros_like(x), torch.round(x / torch.where(s == 0, torch.ones_like(s), s)))
    return torch.clamp(q, -127, 127), s


def _newton(u):
    x = u / (torch.linalg.vector_norm(u) + EPS)
    left = x.shape[0] <= x.shape[1]
    eye = torch.eye(min(x.shape), dtype=torch.float64, device=x.device)
    for _ in range(STEPS):
        gram = torch.mm(x, x.t()) if left else torch.mm(x.t(), x)
        p = COEF[0] * eye + torch.mm(COEF[1] * eye + COEF[2] * gram, gram)
        x = torch.mm(p, x) if left else torch.mm(x, p)
    return x


def exact(case, seed):
    s = prepare(case, seed)
    d = {key: v.double() for key, v in s.items() if isinstance(v, torch.Tensor)}
    kind = case["kind"]
    if kind == "quant":
        q, sc = _scaled(d["src"])
        return {"values": q * sc, "scale": sc[:, 0]}
    if kind == "ortho":
        return torch.stack([_newton(u) for u in d["x"]])
    if kind == "muon":
        v = MU * d["v"] + d["dw"]
        return {"w": (1 - LR * WD) * d["w"] - LR * SCALE * _newton(d["dw"] + MU * v), "v": v}
    m, n, k = case["m"], case["n"], case["k"]
    wq, sw = d["wq"][:, :k], d["sw"][None, :]
    b = d.get("b", torch.zeros((), dtype=torch.float64, device=DEV))
    xq = sx = None
    if kind == "gemm":
        xq, sx = d["xq"][:, :k], d["sx"][:, None]
    elif kind == "bwd":
        xq, sx = d["xqt"][:, :m].t(), d["sx"][:, None]
    else:
        xq, sx = _scaled(d["x"])
    out = {}
    if kind != "bwd":
        y = torch.mm(xq, wq.t()) * (sx * sw) + b
        if kind != "train":
            return y
        out["y"] = y
    # the gradient takes the scale of the summed index with it, as an FP32 number
    gq, sg = _scaled((d["dy"] * sw).float().double())
    out["dx"] = torch.mm(gq, wq) * sg
    gq, sg = _scaled((d["dy"] * sx).float().double().t())
    out["dw"] = torch.mm(gq, xq) * sg
    out["db"] = torch.sum(d["dy"], dim=0)
    return out
