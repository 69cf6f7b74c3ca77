"""The INT8 linear layer and the orthogonalised update in NumPy, from their
definitions: integers exactly, everything else in 64 bits."""
import numpy as np

import oracle


def ld(cols):
    return -(-cols // 128) * 128


def scales(x):
    """FP32 scales of the rows of x (FP32 values), NaN where a row is not finite."""
    with np.errstate(all="ignore"):
        a = np.max(np.abs(x), axis=1).astype(np.float32)
        s = (a / np.float32(127)).astype(np.float32)
    return np.where(np.all(np.isfinite(x), axis=1), s, np.float32(np.nan)).astype(np.float32)


def quantize_rows(x, rounding="nearest", seed=0, role=0, order=None):
    """(q int8 [rows][cols], s FP32 [rows]) of FP32 rows. order: flat index of each element (default row-major)."""
    x = np.asarray(x, np.float32)
    s = scales(x)
    live = s > 0
    s64 = np.where(live, s, 1).astype(np.float64)[:, None]
    x64 = np.where(live[:, None], x, 0).astype(np.float64)
    # the quotient of two FP32 numbers is a tie only if it is one exactly, and 53 bits show that
    q = np.rint(x64 / s64)
    if rounding == "stochastic":
        order = np.arange(x.size).reshape(x.shape) if order is None else order
        e = (x64 - q * s64).astype(np.float32)
        frac = (e / s64.astype(np.float32)).astype(np.float32).astype(np.float64)
        R = np.floor(frac * 2.0 ** 32).astype(np.int64)
        u = np.array([oracle.rng_word(seed, role, int(i)) for i in order.ravel()], np.int64).reshape(x.shape)
        q = q + (R >> 32) + (u < (R & 0xffffffff))
    q = np.clip(q, -127, 127)
    return np.where(live[:, None], q, 0).astype(np.int8), s


def padded(q):
    out = np.zeros((q.shape[0], ld(q.shape[1])), np.int8)
    out[:, :q.shape[1]] = q
    return out


def product(a, sa, b, sb=None, bias=None):
    """64-bit result and the size of what is rounded on the way."""
    y = (a.astype(np.int64) @ b.astype(np.int64).T).astype(np.float64) * sa.astype(np.float64)[:, None]
    if sb is not None:
        y = y * sb.astype(np.float64)[None, :]
    size = np.abs(y)
    if bias is not None:
        y = y + bias.astype(np.float64)[None, :]
    return y, size


def newton_schulz(u, coef, eps):
    """coef: (a, b, c) of every step."""
    x = u.astype(np.float64)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / (np.linalg.norm(x) + eps)
    for a, b, c in coef:
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.T if tall else x
