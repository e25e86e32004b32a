"""oracle/fp8.py against hand-derived values and brute force (CPU)."""
import numpy as np

from oracle import cache as oc
from oracle import fp8 as o8


def test_half_step_is_half_the_distance_between_codes():
    v = np.sort(oc.e4m3_values()[:127])                      # the codes that are not negative, 0 .. 448
    assert v[-1] == 448 and len(v) == 127
    for a, b in zip(v[:-1], v[1:]):
        assert o8.half_step(np.array(a)) == (b - a) / 2


def test_scales_by_hand():
    x = np.zeros((3, 144))
    x[0, 5], x[0, 6], x[0, 130] = -448, 3, 7
    x[1, 0], x[1, 1] = np.inf, 14
    x[2, 143] = np.nan
    tiny = 2.0 ** -120
    assert np.array_equal(o8.scales(x, 1), [[1, 14 / 448, tiny], [7 / 448, tiny, tiny]])
    assert np.array_equal(o8.scales(x, 128), [[1, 7 / 448]])
    assert np.array_equal(o8.per_value(np.array([[1.0, 2, 3], [4, 5, 6]]), (3, 144), 1)[:, [0, 127, 128, 143]],
                          [[1, 1, 4, 4], [2, 2, 5, 5], [3, 3, 6, 6]])


def test_codes_within_half_a_step():
    y, s = np.array([[1.0, 17.0, 0.0, np.nan]]), np.array([[1.0]])
    assert o8.codes_ok(np.array([[1.0, 16.0, 0.0, np.nan]]), y, s, 1, 0.0).all()      # 17 lies in the middle of 16 and 18
    assert o8.codes_ok(np.array([[1.0, 18.0, 0.0, np.nan]]), y, s, 1, 0.0).all()
    assert not o8.codes_ok(np.array([[1.125, 17.0, 0.01, 0.0]]), y, s, 1, 0.0)[0, [0, 2, 3]].any()


def test_norm_of_constant_rows():
    h, y, _ = o8.norm(np.full((2, 16), 3.0), np.full((2, 16), -1.0), np.arange(16.0), 1e-30)
    assert np.all(h == 2) and np.allclose(y, np.arange(16.0))


def test_product_by_a_triple_loop():
    rs = np.random.default_rng(1)
    v = oc.e4m3_values()
    v = v[np.isfinite(v)]
    x, w = rs.choice(v, (3, 144)), rs.choice(v, (130, 144))
    xs, ws = rs.random((2, 3)), rs.random((2, 2))
    y, tol, off = o8.product(x, xs, w, ws)
    assert np.all(off == 0)
    for m, n in ((0, 0), (2, 127), (1, 128), (2, 129)):
        ref = sum(x[m, k] * xs[k // 128, m] * w[n, k] * ws[n // 128, k // 128] for k in range(144))
        assert abs(y[m, n] - ref) <= 1e-9 * tol[m, n] / 2.0 ** -24
    g, _, _ = o8.product(x, xs, w, ws, epilogue=2)
    with np.errstate(over="ignore"):
        assert np.allclose(g[:, 3], y[:, 6] / (1 + np.exp(-y[:, 6])) * y[:, 7])


def test_what_eights_on_a_grid_may_lose():
    """One eight with products 2^10, 1 and six zeros: on a grid of 2^-13 of the largest the 1 may be lost up to 2^-3."""
    x, w = np.zeros((1, 16)), np.ones((1, 16))
    x[0, 0], x[0, 1] = 2.0 ** 8, 1
    w[0, 0] = 4
    one = np.ones((1, 1))
    y, tol, off = o8.product(x, one, w, one, wide=False)
    _, tight, _ = o8.product(x, one, w, one)
    assert y[0, 0] == 1025 and np.isclose(tol[0, 0] - tight[0, 0], 7 * 2.0 ** -3) and np.isclose(off[0, 0], 7 * 2.0 ** -3)
