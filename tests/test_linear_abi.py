"""Refusals of the INT8 linear layer and of the orthogonalised update, checked on
the CPU: every one is an error code (or an exception of the binding) before any
HIP call."""
import ctypes
import math
import os

import pytest
import torch

FAKE = 1 << 20  # never dereferenced


@pytest.fixture(scope="module")
def dl():
    from paper_1802_00930_amd import dfp
    if not os.path.exists(dfp.LIB_PATH):
        pytest.skip("libdfp.so not built")
    return dfp


def p(v):
    return ctypes.c_void_p(v) if v else None


def test_layouts_match_the_header(dl):
    assert ctypes.sizeof(dl.LinearDesc) == 32 and dl.LinearDesc.seed.offset == 24
    assert ctypes.sizeof(dl.OrthoDesc) == 24 + 4 * 48 and dl.OrthoDesc.coef.offset == 24


@pytest.mark.parametrize("cols,ld", [(1, 128), (128, 128), (129, 256), (131071, 131072), (0, 0), (-5, 0),
                                     (2 ** 31 - 256, 2 ** 31 - 256), (2 ** 31 - 255, 0)])
def test_i8_ld(dl, cols, ld):
    assert dl.i8_ld(cols) == ld


def quantize(dl, rows=4, cols=8, type=0, rounding=0, role=0, src=FAKE, q=FAKE, s=FAKE, qt=0):
    return dl.lib().dfp_quantize_i8(rows, cols, type, rounding, 0, role, p(src), p(q), p(s), p(qt), None)


def test_quantize_refusals(dl):
    assert quantize(dl, src=0) == quantize(dl, q=0) == quantize(dl, s=0) == dl.ERR_NULL
    assert quantize(dl, type=3) == quantize(dl, type=-1) == dl.ERR_PARAM
    assert quantize(dl, rounding=2) == quantize(dl, rounding=3) == quantize(dl, rounding=-1) == dl.ERR_PARAM
    assert quantize(dl, role=5) == quantize(dl, role=-1) == dl.ERR_PARAM
    assert quantize(dl, rows=0) == quantize(dl, cols=0) == quantize(dl, cols=2 ** 31) == dl.ERR_SHAPE
    assert quantize(dl, rows=1 << 20, cols=1 << 20) == quantize(dl, rows=(1 << 18) + 1, cols=1 << 18) == dl.ERR_SHAPE
    assert quantize(dl, src=FAKE + 8) == quantize(dl, q=FAKE + 8) == quantize(dl, qt=FAKE + 4) == dl.ERR_ALIGN
    assert quantize(dl, s=FAKE + 2) == dl.ERR_ALIGN


# calls with their pointers by name; the workspace and stream follow
CALLS = {
    "dfp_gemm_i8": ["a", "sa", "b", "sb", "bias", "out"],
    "dfp_linear_i8_fwd": ["x", "wq", "sw", "bias", "y", "xq", "sx", "xqt"],
    "dfp_linear_i8_bwd_data": ["dy", "wqt", "sw", "dx"],
    "dfp_linear_i8_bwd_weights": ["dy", "xqt", "sx", "dw", "db"],
}
OPTIONAL = {"bias", "xq", "xqt", "db"}
SCALES = {"sa", "sb", "sw", "sx", "bias", "db"}
SUMMED = {"dfp_gemm_i8": "k", "dfp_linear_i8_fwd": "k", "dfp_linear_i8_bwd_data": "n",
          "dfp_linear_i8_bwd_weights": "m"}


def call(dl, name, d, ws=FAKE, wsn=1 << 50, **kw):
    ptrs = [p(kw.get(a, FAKE)) for a in CALLS[name]]
    return getattr(dl.lib(), name)(ctypes.byref(d) if d is not None else None, *ptrs, p(ws), wsn, None)


def desc(dl, **kw):
    d = dl.make_linear_desc(4, 8, 16)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("name", list(CALLS))
def test_linear_refusals(dl, name):
    good = desc(dl)
    assert call(dl, name, None) == dl.ERR_NULL
    for a in CALLS[name]:
        optional = a in OPTIONAL or (a == "sx" and name == "dfp_linear_i8_fwd")
        if not optional:
            assert call(dl, name, good, **{a: 0}) == dl.ERR_NULL, a
        assert call(dl, name, good, **{a: FAKE + (2 if a in SCALES else 8)}) == dl.ERR_ALIGN, a
    for field, value in (("type", 3), ("type", -1), ("rounding", 2), ("rounding", 3)):
        assert call(dl, name, desc(dl, **{field: value})) == dl.ERR_PARAM, field
    for field in "mnk":
        for value in (0, -1, 2 ** 26 + 1, 2 ** 31 - 1):
            assert call(dl, name, desc(dl, **{field: value})) == dl.ERR_SHAPE, field
    assert call(dl, name, desc(dl, **{SUMMED[name]: 131072})) == dl.ERR_SHAPE
    assert call(dl, name, desc(dl, m=1 << 20, n=1 << 20)) == dl.ERR_SHAPE
    need = dl.linear_i8_workspace_bytes(good)
    assert call(dl, name, good, ws=0) == call(dl, name, good, wsn=need - 1) == dl.ERR_WORKSPACE
    assert call(dl, name, good, ws=FAKE + 128) == dl.ERR_ALIGN


def test_linear_workspace(dl):
    d = desc(dl, m=300, n=70, k=1000)
    assert dl.linear_i8_workspace_bytes(d) >= 300 * 1024 + 300 * 4
    d.m = 0
    assert dl.linear_i8_workspace_bytes(d) == 0


def ortho(dl, d, x=FAKE, out=FAKE, ws=FAKE, wsn=1 << 50):
    return dl.lib().dfp_orthogonalize(ctypes.byref(d) if d is not None else None, p(x), p(out), p(ws), wsn, None)


def muon(dl, d, w=FAKE, v=FAKE, dw=FAKE, wq=0, sw=0, wqt=0, nesterov=1, ws=FAKE, wsn=1 << 50):
    return dl.lib().dfp_muon_quantize(ctypes.byref(d) if d is not None else None, 0.1, 0.9, 0.0, 1.0, nesterov, p(w),
                                      p(v), p(dw), p(wq), p(sw), p(wqt), p(ws), wsn, None)


def test_ortho_refusals(dl):
    good = dl.make_ortho_desc(2, 30, 40)
    for f in (ortho, muon):
        assert f(dl, None) == dl.ERR_NULL
        for change in (dict(type=3), dict(steps=0), dict(steps=17), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.inf),
                       dict(eps=math.nan)):
            d = dl.make_ortho_desc(2, 30, 40)
            for k, v in change.items():
                setattr(d, k, v)
            assert f(dl, d) == dl.ERR_PARAM, change
        for bad in (math.nan, math.inf, 64.5, -65.0):
            d = dl.make_ortho_desc(2, 30, 40)
            d.coef[4][1] = bad
            assert f(dl, d) == dl.ERR_PARAM
            d.steps = 4  # a step that is not taken is not looked at
            assert f(dl, d, wsn=0) == dl.ERR_WORKSPACE
        for change in (dict(batch=0), dict(rows=0), dict(cols=-1), dict(rows=65537), dict(cols=65537),
                       dict(batch=65536), dict(batch=17, rows=65536, cols=65536)):
            d = dl.make_ortho_desc(2, 30, 40)
            for k, v in change.items():
                setattr(d, k, v)
            assert f(dl, d) == dl.ERR_SHAPE, change
            assert dl.ortho_workspace_bytes(d) == 0
        need = dl.ortho_workspace_bytes(good)
        assert f(dl, good, ws=0) == f(dl, good, wsn=need - 1) == dl.ERR_WORKSPACE
        assert f(dl, good, ws=FAKE + 64) == dl.ERR_ALIGN
    assert ortho(dl, good, x=0) == ortho(dl, good, out=0) == dl.ERR_NULL
    assert ortho(dl, good, x=FAKE + 8) == ortho(dl, good, out=FAKE + 4) == dl.ERR_ALIGN
    for a in ("w", "v", "dw"):
        assert muon(dl, good, **{a: 0}) == dl.ERR_NULL
        assert muon(dl, good, **{a: FAKE + 8}) == dl.ERR_ALIGN
    assert muon(dl, good, wq=FAKE) == muon(dl, good, sw=FAKE) == muon(dl, good, wqt=FAKE) == dl.ERR_NULL
    assert muon(dl, good, wq=FAKE, sw=FAKE, wqt=FAKE) == dl.ERR_PARAM  # a batch has no one transpose
    assert muon(dl, good, nesterov=2) == dl.ERR_PARAM


def test_coefficients_for_each_step(dl):
    d = dl.make_ortho_desc(1, 4, 4, steps=2, coef=[(1.0, 2.0, 3.0), (4.0, 5.0, 6.0)])
    assert [list(d.coef[i]) for i in range(3)] == [[1, 2, 3], [4, 5, 6], [0, 0, 0]]
    with pytest.raises(ValueError):
        dl.make_ortho_desc(1, 4, 4, steps=3, coef=[(1.0, 2.0, 3.0)] * 2)
    with pytest.raises(TypeError):
        dl.make_ortho_desc(1, 4, 4, dtype=torch.float64)
