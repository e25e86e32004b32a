"""Oracle for a decode step over a pruned context: position rotation, the paged cache (16 bits, or
e4m3 codes with a scale for each page and head), attention over it, and 4-bit weights.

TEST INFRASTRUCTURE ONLY: imported by tests, never by the product path.

Everything is float64 numpy, one sequence, page and head at a time.  Tolerances come with the
results where they depend on the data: a rounding is off by at most half a step.
"""
from __future__ import annotations

import math

import numpy as np

E4M3_MAX = 448.0
MIN_EXP = -120


def e4m3_values() -> np.ndarray:
    """The values of the 256 codes (1 sign, 4 exponent, 3 mantissa bits, bias 7, no infinities)."""
    out = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        out[c] = math.nan if e == 15 and m == 7 else (-v if s else v)
    return out


def page_scale(top: float) -> float:
    """The least 2^e, e >= -120, with top <= 448 * 2^e."""
    e = MIN_EXP
    while E4M3_MAX * 2.0 ** e < top:
        e += 1
    return 2.0 ** e


def axis_of(dim: int, sections=None) -> np.ndarray:
    if sections is None:
        return np.zeros(dim // 2, np.int64)
    return np.repeat(np.arange(3), sections)


def rotate(x: np.ndarray, positions: np.ndarray, inv_freq: np.ndarray, sections=None) -> np.ndarray:
    """x [n, heads, dim]; positions [axes, n]; pair (f, f + dim/2) turns by positions[axis] * inv_freq[f]."""
    half = x.shape[-1] // 2
    ang = positions[axis_of(x.shape[-1], sections)].T.astype(np.float64) * inv_freq.astype(np.float64)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def append(pool: np.ndarray, scale, x: np.ndarray, cu, ctx, table, page: int, bits: int):
    """Appends x [n, heads, dim] to pool [pages, heads, page, dim] (values; bits 8: codes' values, with
    scale [pages, heads]).  New entries are NOT rounded (bits 8: x / scale).  Returns (pool, scale, written), written
    a mask of the slots [pages, page] that took a new token."""
    pool = pool.copy()
    scale = None if scale is None else scale.copy()
    written = np.zeros((pool.shape[0], page), bool)
    for b in range(len(ctx)):
        t, r = int(ctx[b]), int(cu[b])
        while r < cu[b + 1]:
            slot, j = t % page, t // page
            n = min(page - slot, cu[b + 1] - r)
            pg = table[b, j] if j < table.shape[1] else -1
            if 0 <= pg < pool.shape[0]:
                part = x[r:r + n]                                  # [n, heads, dim]
                written[pg, slot:slot + n] = True
                for h in range(pool.shape[1]):
                    if bits == 16:
                        pool[pg, h, slot:slot + n] = part[:, h]
                        continue
                    fin = np.abs(part[:, h][np.isfinite(part[:, h])])
                    s = page_scale(fin.max() if fin.size else 0.0)
                    if slot:
                        s = max(s, scale[pg, h])
                        pool[pg, h, :slot] *= scale[pg, h] / s
                    scale[pg, h] = s
                    pool[pg, h, slot:slot + n] = part[:, h] / s
            t, r = t + n, r + n
    return pool, scale, written


def attention(q, k, v, k_scale, v_scale, cu, seq_len, table, page: int, scale: float, window: int = 0, sinks: int = 0):
    """q [n, Hq, d]; k, v [pages, heads, page, d] values (times their scale if given).  Returns (o, lse [Hq, n],
    spread [n, Hq, d], reach [Hq, n]): spread is sum_j P_j |v_j| and reach is scale * max_j sum_d |q_d k_jd| over the
    seen keys, what roundings of P and of the scores act on."""
    n, hq, d = q.shape
    pages, heads = k.shape[:2]
    o, spread = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    lse, reach = np.full((hq, n), -np.inf), np.zeros((hq, n))
    for b in range(len(seq_len)):
        L, nq = int(seq_len[b]), int(cu[b + 1] - cu[b])
        for i in range(nq):
            p, r = L - nq + i, int(cu[b]) + i
            keys = [j for j in range(max(0, p + 1)) if window == 0 or j > p - window or j < sinks]
            keys = [j for j in keys if 0 <= table[b, j // page] < pages]
            if not keys:
                continue
            pg, sl = table[b, [j // page for j in keys]], np.array(keys) % page
            for h in range(hq):
                hk = h // (hq // heads)
                K, V = k[pg, hk, sl], v[pg, hk, sl]
                if k_scale is not None:
                    K, V = K * k_scale[pg, hk][:, None], V * v_scale[pg, hk][:, None]
                s = K @ q[r, h] * scale
                m = s.max()
                if m == -np.inf:
                    continue
                e = np.exp(s - m)
                lse[h, r] = m + math.log(e.sum())
                o[r, h] = e @ V / e.sum()
                spread[r, h] = e @ np.abs(V) / e.sum()
                reach[h, r] = scale * (np.abs(K) @ np.abs(q[r, h])).max()
    return o, lse, spread, reach


def w4_weights(w: np.ndarray, scale: np.ndarray, zero, group: int) -> np.ndarray:
    """W [N, K] from uint8 [N, K/2] (low half first), scale and zero [N, K/group] (zero None: 8)."""
    q = np.empty((w.shape[0], 2 * w.shape[1]))
    q[:, 0::2], q[:, 1::2] = w & 15, w >> 4
    z = np.full(scale.shape, 8.0) if zero is None else zero.astype(np.float64)
    return (q - np.repeat(z, group, 1)) * np.repeat(scale, group, 1)


def w4(x, w, scale, zero, group: int, bias=None, residual=None, epilogue: int = 0):
    """Returns (C, tol): tol bounds what sums in 32 bits may add to the one rounding of the output.  A
    kernel may form sum x (q + 128) and take (zero + 128) sum x off again: terms of at most 143 |x| scale, at most 32
    roundings one after the other in a group (2^-24 each), then one rounding for each group."""
    W = w4_weights(w, scale, zero, group)
    y = x @ W.T
    t = 32 * 2.0 ** -24 * 143 * np.abs(x) @ np.repeat(scale, group, 1).T + \
        (x.shape[1] // group + 2) * 2.0 ** -24 * np.abs(x) @ np.abs(W).T
    if bias is not None:
        y = y + bias
    if epilogue == 1:
        y = y + residual
    if epilogue == 2:
        g, u, tg, tu = y[:, 0::2], y[:, 1::2], t[:, 0::2], t[:, 1::2]
        silu = g / (1 + np.exp(-g))
        # |silu'| <= 1.1; the sigmoid's own arithmetic is a few roundings
        return silu * u, 1.1 * tg * np.abs(u) + np.abs(silu) * tu + 1.1 * tg * tu + 2.0 ** -20 * np.abs(silu * u)
    return y, t + 2.0 ** -22 * np.abs(y)
