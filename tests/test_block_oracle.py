"""The float64 forms of a gated block's operators against brute force: loops over elements,
exact rationals, and differences."""
from fractions import Fraction
import math

import numpy as np
import pytest

from oracle import blocks as K


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_activation(kind):
    g = np.linspace(-9.0, 9.0, 181)
    act, slope = K.activation(g, kind)
    for x, a in zip(g, act):
        part = 1 / (1 + math.exp(-x)) if kind == "silu" else (
            0.5 * math.erfc(-x / math.sqrt(2)))
        assert a == pytest.approx(x * part, rel=1e-14, abs=0)
    h = 1e-5    # differences: the third derivative is below 2, rounding below 1e-15 / h
    up, down = K.activation(g + h, kind)[0], K.activation(g - h, kind)[0]
    np.testing.assert_allclose((up - down) / (2 * h), slope, rtol=0, atol=2e-9)
    # far out: 0 below, the value itself above
    act, slope = K.activation(np.array([-800.0, 800.0]), kind)
    assert act[0] == 0 and act[1] == 800 and slope[0] == 0 and slope[1] == 1


def case(seed):
    rng = np.random.default_rng(seed)
    off = np.array([0, 2, 2, 5])
    return rng, off, rng.standard_normal((6, 3)), rng.standard_normal((3, 8, 3))


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gated_linear(kind):
    rng, off, x, w = case(1)
    h, pre, mag = K.gated_linear(x, w, off, kind)
    for e in range(3):
        for t in range(off[e], off[e + 1]):
            for j in range(4):
                g = sum(x[t, k] * w[e, j, k] for k in range(3))
                u = sum(x[t, k] * w[e, 4 + j, k] for k in range(3))
                assert pre[t, j] == pytest.approx(g, rel=1e-13, abs=1e-15)
                assert pre[t, 4 + j] == pytest.approx(u, rel=1e-13, abs=1e-15)
                assert h[t, j] == pytest.approx(K.activation(np.array(g), kind)[0] * u, rel=1e-12,
                                                abs=1e-15)
    assert (h[5] == 0).all() and (pre[5] == 0).all() and (mag >= np.abs(pre) - 1e-15).all()


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gated_dgrad_is_the_slope_of_the_block(kind):
    rng, off, _, _ = case(2)
    v, pre, dy = rng.standard_normal((3, 5, 4)), rng.standard_normal((6, 8)), rng.standard_normal(
        (6, 5))
    got, of_d = K.gated_dgrad(dy, v, pre, off, kind)

    def loss(p):
        h = K.gated(p, kind)
        return sum(float((dy[t] * (v[e] @ h[t])).sum())
                   for e in range(3) for t in range(off[e], off[e + 1]))
    for t in range(6):
        for j in range(8):
            a, b = pre.copy(), pre.copy()
            a[t, j] += 1e-5
            b[t, j] -= 1e-5
            assert got[t, j] == pytest.approx((loss(a) - loss(b)) / 2e-5, abs=2e-8)
    assert (of_d >= np.abs(got) - 1e-15).all() and (got[5] == 0).all()


def test_layer_norm_in_rationals():
    x = np.array([[1.0, 2.5, -3.0, 0.25, 7.0], [4.0, 4.0, 4.0, 4.0, 4.0]])
    w, b = np.array([1.0, 2.0, -1.0, 0.5, 3.0]), np.array([0.0, 1.0, 0.0, -2.0, 0.5])
    y, mean, rstd = K.layer_norm(x, w, b, 0.125)
    for r in range(2):
        v = [Fraction(float(q)) for q in x[r]]
        m = sum(v) / 5
        var = sum((q - m) ** 2 for q in v) / 5
        s = 1 / math.sqrt(var + Fraction(1, 8))
        assert mean[r] == pytest.approx(float(m)) and rstd[r] == pytest.approx(s, rel=1e-14)
        np.testing.assert_allclose(y[r], [float(q - m) * s * float(p) + float(o)
                                          for q, p, o in zip(v, w, b)], rtol=1e-13)


def test_layer_norm_gradients_are_slopes():
    rng = np.random.default_rng(3)
    x, dy, w, b = (rng.standard_normal(s) for s in ((4, 6), (4, 6), 6, 6))

    def loss(x, w, b):
        return float((K.layer_norm(x, w, b, 1e-3)[0] * dy).sum())
    dx, dw, db = K.layer_norm_backward(dy, x, w, 1e-3)
    for v, d, at in ((x, dx, 0), (w, dw, 1), (b, db, 2)):
        for i in np.ndindex(v.shape):
            p, q = v.copy(), v.copy()
            p[i] += 1e-5
            q[i] -= 1e-5
            args = [[x, w, b], [x, w, b]]
            args[0][at], args[1][at] = p, q
            assert d[i] == pytest.approx((loss(*args[0]) - loss(*args[1])) / 2e-5, abs=5e-8)


def test_clip():
    g = [np.array([3.0, 4.0]), np.array([[12.0]])]
    assert K.clip(g, [], 6.5, 0.0) == (13.0, 0.5)
    assert K.clip(g[1:], [5.0], 13.0, 0.0) == (13.0, 1.0)
    assert K.clip(g, [], 13.0, 13.0) == (13.0, 0.5)
    assert K.clip([], [], 0.0, 0.0) == (0.0, 1.0)
    assert K.clip(g, [math.inf], 1.0, 0.0) == (math.inf, 0.0)
    n, c = K.clip(g, [math.nan], 1.0, 0.0)
    assert math.isnan(n) and math.isnan(c)
