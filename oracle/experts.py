"""Plain float64 forms of the expert step's operators (test infrastructure only).

Rows lie sorted by expert, expert e's in [offsets[e], offsets[e + 1]).  Inputs are
numpy arrays holding the operands' values exactly; outputs are the formulas' values
before their last rounding, with what their rounding errors scale with."""
from __future__ import annotations

import numpy as np


def grouped_rows(rows, weight, offsets):
    """(out, mag): out[t] = rows[t] @ weight[e] for e's rows t (weight: [E, K, N]), 0 for rows
    of nobody; mag = |rows| @ |weight|, the sum of the products' magnitudes."""
    N = weight.shape[2]
    out, mag = np.zeros((len(rows), N)), np.zeros((len(rows), N))
    for e in range(len(weight)):
        a, b = offsets[e], offsets[e + 1]
        r, w = rows[a:b].astype(np.float64), weight[e].astype(np.float64)
        out[a:b] = r @ w
        mag[a:b] = np.abs(r) @ np.abs(w)
    return out, mag


def grouped_wgrad(dy, x, offsets):
    """(dw, mag): dw[e] = dy_e^T x_e and the sums of its products' magnitudes."""
    dw, mag = [], []
    for a, b in zip(offsets[:-1], offsets[1:]):
        p, q = dy[a:b].astype(np.float64), x[a:b].astype(np.float64)
        dw.append(p.T @ q)
        mag.append(np.abs(p).T @ np.abs(q))
    return np.stack(dw), np.stack(mag)


def block_sumsq(dw, block=128):
    """Sums of squares over block x block blocks of each matrix, row-major."""
    out = []
    for w in dw.astype(np.float64):
        out.append([np.sum(w[i:i + block, j:j + block] ** 2)
                    for i in range(0, w.shape[0], block) for j in range(0, w.shape[1], block)])
    return np.array(out)


def row_codes(x):
    """(codes, scale) of the rows of x in the operator's own fp32 arithmetic: it is
    elementwise, so equal bits are expected."""
    x = x.astype(np.float32)
    amax = np.max(np.abs(x), axis=1, initial=0.0)
    bad = ~np.isfinite(x).all(axis=1)
    zero = ~bad & (amax < np.float32(2.0 ** -100))
    safe = np.where(bad | zero, np.float32(1), amax).astype(np.float32)
    inv, scale = np.float32(127) / safe, safe / np.float32(127)
    q = np.rint(np.where(np.isfinite(x), x, 0) * inv[:, None]).astype(np.int64)
    q[bad | zero] = 0
    scale = np.where(bad, np.float32(np.nan), np.where(zero, np.float32(0), scale))
    return q, scale.astype(np.float32)


def quantized_linear(q, sx, codes, sw, offsets):
    """The fp32 value that is rounded to bf16: float(sum) * (sx * sw), the sum exact."""
    y = np.zeros((len(q), codes.shape[1]), np.float32)
    for e in range(len(codes)):
        a, b = offsets[e], offsets[e + 1]
        s = (q[a:b].astype(np.float64) @ codes[e].astype(np.float64).T).astype(np.float32)
        y[a:b] = s * (sx[a:b, None] * sw[e][None, :]).astype(np.float32)
    return y


def orthogonalize(g, steps, coefficients, eps, scale=1.0):
    """Newton-Schulz steps on one matrix, smaller side first."""
    a, b, c = coefficients
    x = g.astype(np.float64)
    flip = x.shape[0] > x.shape[1]
    if flip:
        x = x.T
    x = x / (np.sqrt(np.sum(x * x)) + eps)
    for _ in range(steps):
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    return scale * (x.T if flip else x)


def bf16(x):
    """float32 values rounded to bf16 (nearest even), as float32."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16
    r = np.where(np.isnan(x), np.uint32(0x7FC00000), r)
    return r.astype(np.uint32).view(np.float32)
