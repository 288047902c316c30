"""CPU oracle of the 8-bit floating-point operators, in plain numpy: test infrastructure only.

Values are float64 unless a step is defined in float32 (a block's scale and the unit value that is rounded to 8 bits),
where the float32 operations are done one by one, so that conversions can be compared bit for bit.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
MAX = {"e4m3": 448.0, "e5m2": 57344.0}
MANTISSA = {"e4m3": 3, "e5m2": 2}
LOWEST = {"e4m3": -6, "e5m2": -14}  # exponent of the smallest normal number


def decode_table(fmt):
    """The values of all 256 codes."""
    m, bias = MANTISSA[fmt], 1 - LOWEST[fmt]
    out = np.empty(256)
    for code in range(256):
        sign = -1.0 if code & 128 else 1.0
        e, f = (code & 127) >> m, code & ((1 << m) - 1)
        if fmt == "e4m3" and (code & 127) == 127:
            v = np.nan
        elif fmt == "e5m2" and e == 31:
            v = np.inf if f == 0 else np.nan
        elif e == 0:
            v = f * 2.0 ** (LOWEST[fmt] - m)
        else:
            v = (1 + f / 2.0**m) * 2.0 ** (e - bias)
        out[code] = sign * v
    return out


def round8(u, fmt):
    """Nearest 8-bit value of u, ties to even, magnitudes above MAX to MAX; NaN stays NaN."""
    u = np.asarray(u, dtype=np.float64)
    with np.errstate(invalid="ignore"):
        c = np.clip(u, -MAX[fmt], MAX[fmt])
        e = np.maximum(np.frexp(c)[1] - 1, LOWEST[fmt])
        step = np.ldexp(1.0, e - MANTISSA[fmt])
        return np.round(c / step) * step


def blocks(n):
    return -(-n // BLOCK)


def amax(v, tiles):
    """Largest finite magnitude of each block."""
    rows, cols = v.shape
    a = np.where(np.isfinite(v), np.abs(v), 0.0)
    rb, cb = (blocks(rows) if tiles else rows), blocks(cols)
    out = np.zeros((rb, cb), dtype=v.dtype)
    for i in range(rb):
        for j in range(cb):
            part = a[i * BLOCK:(i + 1) * BLOCK] if tiles else a[i:i + 1]
            part = part[:, j * BLOCK:(j + 1) * BLOCK]
            out[i, j] = part.max()
    return out


def spread(s, rows, cols, tiles):
    s = np.repeat(s, BLOCK, axis=1)[:, :cols]
    return np.repeat(s, BLOCK, axis=0)[:rows] if tiles else s


def quantize(x, tiles=False, pow2=False, fmt="e4m3"):
    """(q values, scales) of a float32 matrix: the float32 steps of the conversion's definition."""
    x = np.asarray(x, dtype=np.float32)
    most = amax(x, tiles)
    s = np.maximum(most / np.float32(MAX[fmt]), np.float32(2.0**-126)).astype(np.float32)
    if pow2:
        m, e = np.frexp(s.astype(np.float64))
        s = np.ldexp(1.0, np.where(m == 0.5, e - 1, e)).astype(np.float32)
        inv = (np.float32(1) / s).astype(np.float32)
    else:
        with np.errstate(divide="ignore", over="ignore"):
            inv = np.minimum(np.float32(MAX[fmt]) / most, np.float32(2.0**126)).astype(np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        u = (x * spread(inv, *x.shape, tiles)).astype(np.float32)
    return round8(np.where(np.isfinite(x), u, np.nan), fmt), s


def dequantize(q, s, tiles=False):
    return np.asarray(q, dtype=np.float64) * spread(np.asarray(s, dtype=np.float64), *q.shape, tiles)


def linear(x, w, bias=None, add=None):
    """(y, sum of the terms' magnitudes) of float64 operands."""
    y, terms = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        y, terms = y + bias, terms + np.abs(bias)
    if add is not None:
        y, terms = y + add, terms + np.abs(add)
    return y, terms


def rmsnorm(h, weight, eps):
    """(h rstd weight, rstd)."""
    rstd = 1.0 / np.sqrt(np.mean(h * h, axis=1) + eps)
    return h * rstd[:, None] * weight, rstd


def rmsnorm_backward(dy, h, rstd, weight, dh=None):
    """(dx, dw, sum of magnitudes in dx, in dw)."""
    x = h * rstd[:, None]
    g = dy * weight
    mean = np.mean(g * x, axis=1, keepdims=True)
    dx = rstd[:, None] * (g - x * mean)
    size = rstd[:, None] * (np.abs(g) + np.abs(x) * np.mean(np.abs(g * x), axis=1, keepdims=True))
    if dh is not None:
        dx, size = dx + dh, size + np.abs(dh)
    return dx, np.sum(dy * x, axis=0), size, np.sum(np.abs(dy * x), axis=0)


def sigmoid(g):
    return 0.5 * (1.0 + np.tanh(0.5 * g))


def gated(g, u):
    return g * sigmoid(g) * u


def gated_backward(g, u, da):
    """(dg, du, magnitude of dg's terms, of du)."""
    sig = sigmoid(g)
    dg = da * u * sig * (1.0 + g * (1.0 - sig))
    return dg, da * g * sig, np.abs(da * u) * sig * (1.0 + np.abs(g) * (1.0 - sig)), np.abs(da * g * sig)


def halves(g, u):
    """g and u side by side, the up half from the next multiple of 128."""
    up = blocks(g.shape[1]) * BLOCK
    out = np.zeros((g.shape[0], up + g.shape[1]), dtype=g.dtype)
    out[:, :g.shape[1]] = g
    out[:, up:] = u
    return out


def rounding_bound(v, s, fmt="e4m3"):
    """How far an 8-bit value may be from v for rounding alone: half a step of v's binade, which is at most |v| over
    2^(mantissa + 1), or half the subnormal step times the scale."""
    m = MANTISSA[fmt]
    return np.maximum(np.abs(v) * 2.0 ** -(m + 1), s * 2.0 ** (LOWEST[fmt] - m - 1))
