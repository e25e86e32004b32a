"""Pins of oracle/cache.py against closed forms and independent routines (CPU)."""
import math

import numpy as np
import pytest

from oracle import attention as oatt
from oracle import cache as oc


def test_e4m3_table_is_torchs():
    torch = pytest.importorskip("torch")
    v = torch.arange(256, dtype=torch.int64).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(v), np.isnan(oc.e4m3_values()))
    assert np.array_equal(v[~np.isnan(v)], oc.e4m3_values()[~np.isnan(v)])


def test_page_scale():
    assert oc.page_scale(448.0) == 1.0 and oc.page_scale(448.1) == 2.0 and oc.page_scale(224.0) == 0.5
    assert oc.page_scale(0.0) == 2.0 ** -120


def test_rotation_is_complex_multiplication():
    rs = np.random.default_rng(0)
    x, pos = rs.standard_normal((5, 3, 80)), rs.integers(0, 1000, (3, 5))
    freq = (100.0 ** (-np.arange(40) / 40)).astype(np.float32)
    y = oc.rotate(x, pos, freq, (8, 16, 16))
    for f in range(40):
        a = pos[0 if f < 8 else 1 if f < 24 else 2] * float(freq[f])
        z = (x[..., f] + 1j * x[..., f + 40]) * np.exp(1j * a)[:, None]
        assert np.allclose(y[..., f], z.real) and np.allclose(y[..., f + 40], z.imag)
    # scores depend on the distance of two positions alone
    one = np.ones((1, 1, 80))
    s = [(oc.rotate(one, np.array([[7 + t]]), freq) * oc.rotate(one, np.array([[t]]), freq)).sum() for t in (0, 50)]
    assert s[0] == pytest.approx(s[1])


def test_append_then_attention_is_causal_attention():
    """Pages filled in two calls hold what was appended; attention over them is the causal oracle's."""
    rs = np.random.default_rng(1)
    n, hq, hkv, d, page = 45, 4, 2, 80, 16
    q, k, v = rs.standard_normal((n, hq, d)), rs.standard_normal((n, hkv, d)), rs.standard_normal((n, hkv, d))
    table = np.array([[4, 0, 2]])
    pool = [np.full((5, hkv, page, d), np.nan) for _ in range(2)]
    for a, b in ((0, 20), (20, 45)):
        pool = [oc.append(p, None, x[a:b], [0, b - a], [a], table, page, 16)[0] for p, x in zip(pool, (k, v))]
    o, lse, spread, _ = oc.attention(q, pool[0], pool[1], None, None, [0, n], [n], table, page, 0.1)
    O, L, _ = oatt.attention_segment(q, k, v, True, 0.1)
    assert np.allclose(o, O) and np.allclose(lse, L) and np.all(spread >= np.abs(o) - 1e-12)


def test_append_moves_old_codes_to_a_larger_scale():
    table, x = np.array([[0]]), np.zeros((1, 1, 80))
    pool, scale = np.zeros((1, 1, 16, 80)), np.array([[0.25]])
    pool[0, 0, 0] = 96.0
    x[0, 0, 3] = 448.0
    p, s, w = oc.append(pool, scale, x, [0, 1], [1], table, 16, 8)
    assert s[0, 0] == 1.0 and p[0, 0, 0, 0] == 24.0 and p[0, 0, 1, 3] == 448.0 and w.sum() == 1
    p, s, _ = oc.append(pool, scale, x, [0, 1], [0], table, 16, 8)       # a fresh page forgets its scale
    assert s[0, 0] == 1.0 and p[0, 0, 0, 3] == 448.0


def test_window_and_sinks():
    """Equal scores: o is the mean of the seen values, lse the logarithm of their number."""
    d, page, L = 80, 16, 40
    v = np.zeros((3, 1, page, d))
    v[:, 0, :, 0] = np.arange(48).reshape(3, page)
    for window, sinks, seen in ((0, 0, range(40)), (8, 0, range(32, 40)), (8, 3, [0, 1, 2] + list(range(32, 40))),
                                (8, 36, range(40)), (100, 2, range(40))):
        o, lse, _, _ = oc.attention(np.zeros((1, 1, d)), np.zeros_like(v), v, None, None, [0, 1], [L], np.array([[0, 1, 2]]), page,
                                    1.0, window, sinks)
        assert o[0, 0, 0] == pytest.approx(np.mean(list(seen))) and lse[0, 0] == pytest.approx(math.log(len(list(seen))))
    o, lse, _, _ = oc.attention(np.zeros((2, 1, d)), np.zeros_like(v), v, None, None, [0, 2], [1], np.array([[0, 1, 2]]), page, 1.0)
    assert lse[0, 0] == -np.inf and np.all(o[0] == 0) and lse[0, 1] == 0       # the first query is before the first token


def test_w4_by_hand():
    w = np.array([[0x10, 0xF8]] * 1, np.uint8).repeat(16, 0).reshape(1, 32)[:, :16]
    W = oc.w4_weights(w, np.array([[0.5]]), None, 32)
    assert W.shape == (1, 32) and list(W[0, :4]) == [-4.0, -3.5, 0.0, 3.5]
    W = oc.w4_weights(w, np.array([[0.5]]), np.array([[1]], np.uint8), 32)
    assert list(W[0, :4]) == [-0.5, 0.0, 3.5, 7.0]
    x = np.ones((1, 32))
    y, _ = oc.w4(x, np.concatenate([w, w]), np.full((2, 1), 0.5), None, 32, epilogue=2)
    g = 8 * (-4 - 3.5 + 0 + 3.5)
    assert y[0, 0] == pytest.approx(g / (1 + math.exp(-g)) * g)
