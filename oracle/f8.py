"""Definitions of the 8-bit floating-point operators in fp64 numpy -- TEST INFRASTRUCTURE.

e4m3 codes with one scale for each row (of weights: 128 rows) and 128 columns, the norm and the gate before them, the linear
layer behind them.  Written from the formulas; shares nothing with the CUDA library.
"""
from __future__ import annotations

import numpy as np

BLOCK, TOP, MIN_SCALE = 128, 448.0, 2.0 ** -100


def decode(codes):
    """Real values of e4m3 codes (uint8): one sign, four exponent (bias 7), three mantissa bits; 0x7f and 0xff are NaN."""
    c = np.asarray(codes).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    value = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    value = np.where((c & 127) == 127, np.nan, value)
    return np.where(c & 128, -value, value)


def half_step(q):
    """Half the distance between the e4m3 values around |q| <= 448, the larger one at a power of two."""
    e = np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** -6)))
    return 2.0 ** (e - 4)


def scales(v, rows=1):
    """[ceil(n / rows)][ceil(k / 128)] scales of v [n][k]."""
    n, k = v.shape
    out = np.zeros((-(-n // rows), -(-k // BLOCK)))
    for i in range(out.shape[0]):
        for j in range(out.shape[1]):
            cut = np.abs(v[i * rows:(i + 1) * rows, j * BLOCK:(j + 1) * BLOCK])
            cut = cut[np.isfinite(cut)]
            out[i, j] = max(cut.max() / TOP if cut.size else 0.0, MIN_SCALE)
    return out


def spread(s, n, k, rows=1):
    """The scale of every element of [n][k]."""
    return s[np.arange(n) // rows][:, np.arange(k) // BLOCK]


def rmsnorm(x, gain, eps, residual=None):
    """(sum, values) of the rows of x."""
    h = x.astype(np.float64) if residual is None else x.astype(np.float64) + residual.astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        return h, h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps) * gain.astype(np.float64)


def gated(x, gate):
    g = gate.astype(np.float64)
    with np.errstate(over="ignore"):
        return x.astype(np.float64) * (g / (1.0 + np.exp(-g)))


def linear(x_codes, x_scales, w_codes, w_scales, bias=None):
    """(y, sum of the products' magnitudes)."""
    n, k = w_codes.shape
    x = decode(x_codes) * spread(x_scales.astype(np.float64), x_codes.shape[0], k)
    w = decode(w_codes) * spread(w_scales.astype(np.float64), n, k, BLOCK)
    b = np.zeros(n) if bias is None else bias.astype(np.float64)
    return x @ w.T + b, np.abs(x) @ np.abs(w).T + np.abs(b)
