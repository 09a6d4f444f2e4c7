"""Plain float64 forms of a gated block's operators (test infrastructure only): gated
feed-forward by expert, layer norm, clipping by the global norm.

Inputs are numpy arrays holding the operands' values exactly; outputs are the formulas'
values before their last rounding, with what their rounding errors scale with."""
from __future__ import annotations

import math

import numpy as np

from .experts import grouped_rows

_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def activation(g, kind):
    """(act, act') at g."""
    with np.errstate(over="ignore"):
        if kind == "silu":
            s = 1.0 / (1.0 + np.exp(-g))
            return g * s, s * (1.0 + g / (1.0 + np.exp(g)))
        phi = 0.5 * _erfc(-g / math.sqrt(2.0))
        return g * phi, phi + g * np.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)


def gated(pre, kind):
    """h from the products pre = [gate, up]."""
    g, u = np.split(np.asarray(pre, np.float64), 2, axis=1)
    return activation(g, kind)[0] * u


def gated_linear(x, w, offsets, kind):
    """(h, pre, mag): w is [E, 2 H, K]; mag the sums of the products' magnitudes."""
    pre, mag = grouped_rows(x, w.transpose(0, 2, 1), offsets)
    return gated(pre, kind), pre, mag


def gated_dgrad(dy, w, pre, offsets, kind):
    """(dpre, of_d): w is [E, K, H]; of_d what dpre changes by with an error of all d that is the
    sum of their products' magnitudes."""
    d, mag = grouped_rows(dy, w, offsets)
    g, u = np.split(np.asarray(pre, np.float64), 2, axis=1)
    act, slope = activation(g, kind)
    at = np.concatenate([slope * u, act], 1)
    out, of_d = np.concatenate([d, d], 1) * at, np.concatenate([mag, mag], 1) * np.abs(at)
    out[offsets[-1]:] = 0
    of_d[offsets[-1]:] = 0
    return out, of_d


def layer_norm(x, weight, bias, eps):
    """(y, mean, rstd)."""
    x = x.astype(np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    y = y * (1.0 if weight is None else weight.astype(np.float64))
    return y + (0.0 if bias is None else bias.astype(np.float64)), mean, rstd


def layer_norm_backward(dy, x, weight, eps):
    """(dx, dweight, dbias) at the exact statistics of x."""
    dy, (z, _, rstd) = dy.astype(np.float64), layer_norm(x, None, None, eps)
    g = dy * (1.0 if weight is None else weight.astype(np.float64))
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - z * (g * z).mean(1, keepdims=True))
    return dx, (dy * z).sum(0), dy.sum(0)


def clip(gradients, norms, max_norm, eps):
    """(norm, factor): `gradients` those whose squares `norms` does not hold."""
    squares = [float(v) ** 2 for v in norms] + [
        math.fsum((g.astype(np.float64).ravel() ** 2).tolist()) for g in gradients]
    norm = math.sqrt(math.fsum(squares)) if all(map(math.isfinite, squares)) else math.sqrt(
        sum(squares))
    return norm, max_norm / (norm + eps) if norm + eps > max_norm else (
        1.0 if norm == norm else math.nan)
