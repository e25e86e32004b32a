"""Oracle for a layer's 8-bit operators: e4m3 codes with a scale for each block of 128, RMS norm with the residual's
addition, and products of such codes.

TEST INFRASTRUCTURE ONLY: imported by tests, never by the product path.

Everything is float64 numpy.  Values that are stored in fewer bits come unrounded, and tolerances with the results where they
depend on the data: a rounding is off by at most half a step.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128
E4M3_MAX = 448.0
MIN_SCALE = 2.0 ** -120


def half_step(v: np.ndarray) -> np.ndarray:
    """Half the distance between neighbouring e4m3 codes at v: 3 mantissa bits, the least normal exponent -6."""
    e = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
    return 2.0 ** (e - 4)


def blocks(n: int) -> int:
    return -(-n // BLOCK)


def spread(scale: np.ndarray, shape, rows: int) -> np.ndarray:
    """The scale of every value: scale [K blocks, M] for rows = 1, [row blocks, K blocks] for 128."""
    s = scale.T if rows == 1 else np.repeat(scale, rows, 0)
    return np.repeat(s, BLOCK, 1)[:shape[0], :shape[1]]


def scales(x: np.ndarray, rows: int) -> np.ndarray:
    """max(largest finite |x| / 448, 2^-120) of each block, laid out as the library does."""
    M, K = x.shape
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    out = np.empty((blocks(M) if rows > 1 else M, blocks(K)))
    for i in range(out.shape[0]):
        for j in range(out.shape[1]):
            out[i, j] = max(a[i * rows:(i + 1) * rows, j * BLOCK:(j + 1) * BLOCK].max() / E4M3_MAX, MIN_SCALE)
    return out.T.copy() if rows == 1 else out


def codes_ok(got: np.ndarray, y: np.ndarray, scale: np.ndarray, rows: int, tol) -> np.ndarray:
    """Which codes (as values) lie within half a step of y / scale, for the scales that came with them; y known to `tol`,
    and quantised through the scale's reciprocal in 32 bits (three roundings: 2^-22)."""
    s = spread(scale, y.shape, rows)
    with np.errstate(invalid="ignore"):
        v, t = y / s, tol / s
        near = np.abs(got - v) <= half_step(np.abs(v) * (1 + 2.0 ** -22) + t) + t + 2.0 ** -22 * np.abs(v)
    return np.where(np.isfinite(y), near, np.isnan(got))


def norm(x: np.ndarray, residual, gamma: np.ndarray, eps: float):
    """(h, y, tol): tol bounds the 32-bit arithmetic of y.  At most 64 squares of a thread are added one after the other, then 16
    sums of threads: 2^-24 each, halved by the root; h, the mean, eps, the root, the division and two products round once."""
    h = x if residual is None else x + residual
    y = h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * gamma
    return h, y, (0.5 * 80 + 8) * 2.0 ** -24 * np.abs(y)


def product(x, xs, w, ws, bias=None, residual=None, epilogue: int = 0):
    """(C, tol) of code values x [M, K], w [N, K] with their scales.  A block's 128 products are exact and summed by the
    matrix cores: at most 128 steps that each lose less than 2^-23 of the magnitudes' sum; blocks, their scales' product, up to 64
    parts of K and bias or residual round once each (2^-24)."""
    X, W = x * spread(xs, x.shape, 1), w * spread(ws, w.shape, BLOCK)
    y = X @ W.T
    t = (128 * 2.0 ** -23 + (blocks(x.shape[1]) + 68) * 2.0 ** -24) * (np.abs(X) @ np.abs(W).T)
    if bias is not None:
        y = y + bias
        t = t + 2.0 ** -24 * np.abs(y)
    if epilogue == 1:
        y = y + residual
        t = t + 2.0 ** -24 * np.abs(y)
    if epilogue == 2:
        g, u, tg, tu = y[:, 0::2], y[:, 1::2], t[:, 0::2], t[:, 1::2]
        with np.errstate(over="ignore"):
            silu = g / (1 + np.exp(-g))
        # |silu'| <= 1.1; the sigmoid's own arithmetic is a few roundings
        return silu * u, 1.1 * tg * np.abs(u) + np.abs(silu) * tu + 1.1 * tg * tu + 2.0 ** -20 * np.abs(silu * u)
    return y, t
