"""K8 with coefficients that take A = X X^T and the polynomial past what fp16 holds at the
usual scale, and updates whose norm lies far below eps, against the formulas in float64.

Tolerance.  The updates have rows that are orthogonal and equally long (one row, or some of
a Hadamard matrix), so that A = s I and every step multiplies X by p(s): with u = 2^-11
(half a unit in fp16's last place; fp32 sums of at most 512 products stay far below) and e
X's relative error so far, A is off by 2 e + u, p by (|b| s + 2 |c| s^2) (2 e + u) / |p| + u
and X by the sum of that, e and u; the result is rounded once more, by 2^-8."""
import numpy as np
import pytest

from gpu_util import require_gpu
from oracle import experts as X

pytestmark = pytest.mark.gpu
U = 2.0 ** -11


def updates(m, n):
    if m == 1:
        return np.random.default_rng(n).standard_normal((1, n)).astype(np.float32)
    h = np.array([[1.0]])
    while len(h) < n:
        h = np.block([[h, h], [h, -h]])
    return h[:m].astype(np.float32)


def bound(s, coefficients, steps):
    a, b, c = coefficients
    e = U
    for k in range(steps):
        p = a + b * s + c * s * s
        e += (abs(b) * s + 2 * abs(c) * s * s) * (2 * e + U) / abs(p) + U
        if k + 1 < steps:
            e += U
        s *= p * p
    return e + 2.0 ** -8


def run(g, coefficients, steps, eps, dtype=None):
    torch = require_gpu()
    from paper_2606_00539_amd import torch_ops

    print("orthogonalize", g.shape, coefficients, steps, eps, flush=True)
    gt = torch.from_numpy(g).cuda()
    y = torch_ops.orthogonalize(gt if dtype is None else gt.to(dtype), steps=steps,
                                coefficients=coefficients, eps=eps)
    return y.double().cpu().numpy()


# singular values and |p| by step: 1 -> 5 -> 1; 1 with |p(0)| = 20; 1 -> 15 -> -1.9e7; 0.125 ->
# 4.5 -> 162 with p = 36; 0.125 -> 2.5 -> 9.5 -> -2,053; 1 -> 15 -> 15
@pytest.mark.parametrize("coefficients,steps,shape", [
    ((5.2, -0.2, 0.0), 2, (1, 1)),
    ((5.2, -0.2, 0.0), 2, (1, 300)),
    ((5.2, -0.2, 0.0), 2, (300, 1)),
    ((20.0, -19.0, 0.0), 1, (1, 37)),
    ((40.0, 0.0, -25.0), 2, (1, 128)),
    ((36.0, 0.0, 0.0), 2, (64, 128)),
    ((36.0, 0.0, 0.0), 2, (256, 64)),
    ((20.0, -2.6, 0.0), 3, (64, 64)),
    ((15.0625, -0.0625, 0.0), 2, (1, 72)),
])
def test_large_coefficients(coefficients, steps, shape):
    m, n = min(shape), max(shape)
    g = updates(m, n)
    want = X.orthogonalize(g, steps, coefficients, 0.0)
    limit = bound(1.0 / m, coefficients, steps)
    g, want = (g, want) if shape[0] <= shape[1] else (g.T.copy(), want.T)
    got = run(g, coefficients, steps, 0.0)
    assert np.isfinite(got).all()
    assert np.abs(got - want).max() <= limit * np.abs(want).max(), limit


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 300), (300, 1), (64, 128), (256, 64)])
@pytest.mark.parametrize("length,eps,steps", [
    (1e-3, 1e-4, 1), (1e-7, 1e-7, 1), (1e-9, 1e-7, 1), (1e-30, 1.0, 1), (1e-13, 1e-7, 5),
    (1e-25, 1e-7, 5), (1e-30, 1.0, 5), (1e-36, 1e-3, 5)])
def test_norm_below_eps(length, eps, shape, steps, dtype):
    """X = G / (|G| + eps) is small then, and grows by a = 3.4445 a step."""
    torch = require_gpu()
    m, n = min(shape), max(shape)
    g = updates(m, n)
    g = (g * (length / np.linalg.norm(g))).astype(np.float32)
    if dtype == "bf16":
        g = X.bf16(g)
    coefficients = (3.4445, -4.775, 2.0315)
    want = X.orthogonalize(g, steps, coefficients, float(np.float32(eps)))
    s = (np.linalg.norm(g.astype(np.float64)) / (np.linalg.norm(g.astype(np.float64)) + eps)) ** 2
    limit = bound(s / m, coefficients, steps)
    g, want = (g, want) if shape[0] <= shape[1] else (g.T.copy(), want.T)
    got = run(g, coefficients, steps, eps, torch.bfloat16 if dtype == "bf16" else None)
    assert np.abs(want).max() > 1e-37
    assert np.abs(got - want).max() <= limit * np.abs(want).max(), limit
