"""The plain forms of the expert step's operators against independent ones: sums
written out, differences for the gradients, singular values for the
orthogonalisation.  CPU only."""
import numpy as np
import pytest

from oracle import experts as X


def _data(seed, rows=13, E=3, N=5, K=7):
    rng = np.random.default_rng(seed)
    off = np.array([0, 4, 4, 11])          # an expert without rows, two rows of nobody
    return rng, off, rng.standard_normal((rows, K)), rng.standard_normal((E, N, K))


def test_grouped_rows_written_out():
    _, off, x, w = _data(0)
    y, mag = X.grouped_rows(x, w.transpose(0, 2, 1), off)
    for t in range(13):
        owner = [e for e in range(3) if off[e] <= t < off[e + 1]]
        for n in range(5):
            want = sum(x[t, k] * w[owner[0], n, k] for k in range(7)) if owner else 0.0
            assert abs(y[t, n] - want) < 1e-12
            assert mag[t, n] >= abs(want) - 1e-12


@pytest.mark.parametrize("which", ["x", "w"])
def test_gradients_against_differences(which):
    """d/dx and d/dw of sum(y * dy): the formulas of dgrad and wgrad against central
    differences (the function is linear in each, so only rounding is left)."""
    rng, off, x, w = _data(1)
    dy = rng.standard_normal((13, 5))
    dy[11:] = 0.0                          # rows of nobody have no gradient
    f = lambda: float(np.sum(X.grouped_rows(x, w.transpose(0, 2, 1), off)[0] * dy))
    if which == "x":
        got, at = X.grouped_rows(dy, w, off)[0], x
    else:
        got, at = X.grouped_wgrad(dy, x, off)[0], w
    num = np.zeros_like(at)
    for i in np.ndindex(at.shape):
        old, h = at[i], 1e-3
        at[i] = old + h
        hi = f()
        at[i] = old - h
        num[i] = (hi - f()) / (2 * h)
        at[i] = old
    np.testing.assert_allclose(got, num, atol=1e-9)


def test_block_sums_cover_every_value_once():
    rng = np.random.default_rng(2)
    dw = rng.standard_normal((2, 130, 257))
    s = X.block_sumsq(dw)
    assert s.shape == (2, 2 * 3)
    np.testing.assert_allclose(s.sum(1), (dw ** 2).sum((1, 2)), rtol=1e-12)
    np.testing.assert_allclose(s[1, 5], (dw[1, 128:, 256:] ** 2).sum(), rtol=1e-12)


def test_row_codes():
    x = np.array([[1.0, -2.0, 0.5, 127.0], [0.0, 0.0, 0.0, 0.0], [2.0 ** -101, 0, 0, 0],
                  [np.inf, 1, 1, 1], [np.nan, 1, 1, 1], [3.0, -3.0, 1.5, 0.011]], np.float32)
    q, s = X.row_codes(x)
    assert q[0].tolist() == [1, -2, 0, 127] and s[0] == 1.0     # 0.5 goes to the even 0
    assert not q[1:5].any()
    assert s[1] == 0 and s[2] == 0 and np.isnan(s[3]) and np.isnan(s[4])
    assert q[5].tolist() == [127, -127, 64, 0]                  # 63.5 to the even 64


@pytest.mark.parametrize("m,n", [(8, 8), (5, 12), (12, 5)])
def test_orthogonalize_against_the_singular_values(m, n):
    """X = U f(S) V^T with f the scalar polynomial iterated."""
    g = np.random.default_rng(3).standard_normal((m, n))
    u, s, vt = np.linalg.svd(g, full_matrices=False)
    a, b, c = 3.4445, -4.7750, 2.0315
    s = s / (np.linalg.norm(g) + 1e-7)
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    want = 0.5 * (u * s) @ vt
    np.testing.assert_allclose(X.orthogonalize(g, 5, (a, b, c), 1e-7, 0.5), want, atol=1e-9)
    assert np.all(np.abs(s - 1) < 0.35)


def test_bf16_rounds_to_nearest_even():
    x = np.array([1.0, 1.0 + 2.0 ** -8, 1.0 + 3 * 2.0 ** -8, 1.0 + 2.0 ** -8 + 2.0 ** -20],
                 np.float32)
    assert X.bf16(x).tolist() == [1.0, 1.0, 1.0 + 2.0 ** -6, 1.0 + 2.0 ** -7]
