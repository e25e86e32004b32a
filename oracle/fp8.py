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


def per_value(scale: np.ndarray, shape, rows: int) -> np.ndarray:
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
    and divided in 32 bits (2^-22 is ample for the quotient's rounding)."""
    s = per_value(scale, y.shape, rows)
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


def eight_max(x: np.ndarray) -> np.ndarray:
    """The largest magnitude of each 8 neighbouring values of a row."""
    return np.abs(x).reshape(x.shape[0], -1, 8).max(2)


def product(x, xs, w, ws, bias=None, residual=None, epilogue: int = 0, wide: bool = True):
    """(C, tol, spread) of code values x [M, K], w [N, K] with their scales.
    tol bounds what the sums may be off.  Products of two codes are exact (8 bits).  wide: 128 steps of a block that each lose less
    than 2^-23 of the magnitudes' sum.  Not wide: the matrix cores put the products of 8 neighbouring k's on a grid of 2^-13 of
    the largest of them, so that each of the other 7 loses less than that; the eights are added in 32 bits as above.  Blocks, their
    scales' product, up to 64 parts of K and bias or residual round once each (2^-24).
    spread: the eights' part of tol as if they were off in signs of their own, the root of the sum of their squares (0 where wide)."""
    X, W = x * per_value(xs, x.shape, 1), w * per_value(ws, w.shape, BLOCK)
    y = X @ W.T
    t = (128 * 2.0 ** -23 + (blocks(x.shape[1]) + 68) * 2.0 ** -24) * (np.abs(X) @ np.abs(W).T)
    off = np.zeros_like(y)
    if not wide:
        a, b = eight_max(X) * 7 * 2.0 ** -13, eight_max(W)
        t = t + a @ b.T
        off = np.sqrt((a * a) @ (b * b).T)
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
        through = lambda a, b: 1.1 * a * np.abs(u) + np.abs(silu) * b + 1.1 * a * b   # noqa: E731
        return silu * u, through(tg, tu) + 2.0 ** -20 * np.abs(silu * u), through(off[:, 0::2], off[:, 1::2])
    return y, t, off
