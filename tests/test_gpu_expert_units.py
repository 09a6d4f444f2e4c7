"""ExpertUnits and OrthogonalMomentum (torch_experts.py), and the example that trains
with them: outputs by path, gradients against the formulas and against differences, the
controller's norms, accumulation, refusals."""
import os
import sys

import numpy as np
import pytest

from gpu_util import require_gpu
from oracle import experts as X

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def setup(seed, E=4, o=136, i=72, counts=(40, 0, 77, 3), pad=6, **kw):
    torch = require_gpu()
    from paper_2606_00539_amd.torch_experts import ExpertUnits

    rng = np.random.default_rng(seed)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rows = int(off[-1]) + pad
    x = X.bf16(rng.standard_normal((rows, i)).astype(np.float32))
    w = X.bf16((rng.standard_normal((E, o, i)) / np.sqrt(i)).astype(np.float32))
    dy = X.bf16((1e-2 * rng.standard_normal((rows, o))).astype(np.float32))
    dev = lambda a: torch.from_numpy(a).to(torch.bfloat16).cuda()
    weight = torch.nn.Parameter(dev(w))
    units = ExpertUnits([("m", weight)], max_o=2, lock_len=1, **kw)
    return torch, units, weight, off, torch.from_numpy(off).cuda(), x, w, dy, dev


def close(got, want, mag, K, rounded=True):
    slack = (K + 1) * 2.0 ** -23 * mag + (2.0 ** -8 * np.abs(want) if rounded else 0)
    assert (np.abs(got - want) <= slack).all()


def test_both_paths_by_the_mask():
    torch, units, weight, off, d_off, x, w, _, dev = setup(1)
    q, sx = X.row_codes(x)
    c, sw = X.row_codes(w.reshape(-1, w.shape[2]))
    low = X.bf16(X.quantized_linear(q, sx, c.reshape(w.shape), sw.reshape(w.shape[:2]), off))
    high, mag = X.grouped_rows(x, w.transpose(0, 2, 1), off)
    for mask in ([0, 0, 0, 0], [1, 0, 1, 0], [0, 1, 0, 1], [1, 1, 1, 1]):
        units.mask(0).copy_(torch.tensor(mask, dtype=torch.uint8, device="cuda"))
        y = units.linear("m", dev(x), d_off).detach().float().cpu().numpy()
        assert (y[off[-1]:] == 0).all()
        for e in range(4):
            s = slice(off[e], off[e + 1])
            if mask[e]:
                close(y[s], high[s], mag[s], x.shape[1])
            else:
                assert np.array_equal(y[s], low[s])
    units.close()


@pytest.mark.parametrize("grad_dtype", ["f32", "bf16"])
def test_gradients_norms_and_accumulation(grad_dtype):
    torch = require_gpu()
    dt = torch.float32 if grad_dtype == "f32" else torch.bfloat16
    torch, units, weight, off, d_off, x, w, dy, dev = setup(2, grad_dtype=dt)
    total, mags = 0.0, 0.0
    for k in range(3):
        xt = dev(np.roll(x, k, axis=1)).requires_grad_()
        units.linear("m", xt, d_off).backward(dev(dy))
        dx, mag = X.grouped_rows(dy, w, off)
        close(xt.grad.float().cpu().numpy(), dx, mag, w.shape[1])
        dw, mw = X.grouped_wgrad(dy, np.roll(x, k, axis=1), off)
        total, mags = total + dw, mags + mw
    got = units.grads["m"].float().cpu().numpy()
    assert weight.grad is None
    # three sums, in bf16 three roundings of what is held by then
    slack = (max(np.diff(off)) + 3) * 2.0 ** -23 * mags + (3 * 2.0 ** -8 * mags
                                                            if grad_dtype == "bf16" else 0)
    assert (np.abs(got - total) <= slack).all()
    units.step(1.1, 1.5)
    norm = units.query()["norm"]
    np.testing.assert_allclose(norm, np.sqrt((got.astype(np.float64) ** 2).sum((1, 2))), rtol=1e-5)
    assert norm[1] == 0.0                       # the expert without rows
    # after the step a backward starts anew
    units.linear("m", dev(x).requires_grad_(), d_off).backward(dev(dy))
    dw, mw = X.grouped_wgrad(dy, x, off)
    close(units.grads["m"].float().cpu().numpy(), dw, mw, max(np.diff(off)), grad_dtype == "bf16")
    units.close()


@pytest.mark.parametrize("how", ["sum over rows", "sum", "transposed", "part of a vector",
                                 "part of rows"])
def test_gradients_from_any_layout_of_dy(how):
    """The output's gradient as autograd brings it: broadcast rows, broadcast values, columns
    first, contiguous at an odd address, rows an odd number of values apart."""
    torch, units, weight, off, d_off, x, w, _, dev = setup(6, low_cost=False)
    rng = np.random.default_rng(60)
    o = w.shape[1]
    g = X.bf16(rng.standard_normal((len(x), o)).astype(np.float32))
    xt = dev(x).requires_grad_()
    y = units.linear("m", xt, d_off)
    if how == "sum over rows":
        g[:] = g[:1]
        y.sum(0).backward(dev(g[0]))
    elif how == "sum":
        g[:] = 1.0
        y.sum().backward()
    elif how == "transposed":
        y.t().contiguous().backward(dev(g).t().contiguous())
    elif how == "part of a vector":
        torch.cat([y.new_zeros(3), y.flatten()]).backward(
            dev(np.pad(g.ravel(), (3, 0))))
    else:
        torch.cat([y.new_zeros(len(x), 8), y, y.new_zeros(len(x), 1)], 1).backward(
            dev(np.pad(g, ((0, 0), (8, 1)))))
    dx, mag = X.grouped_rows(g, w, off)
    close(xt.grad.float().cpu().numpy(), dx, mag, o)
    dw, mw = X.grouped_wgrad(g, x, off)
    close(units.grads["m"].cpu().numpy(), dw, mw, max(np.diff(off)), rounded=False)
    units.close()


def test_gradients_against_differences():
    """Without the low-cost path the function is linear in x and in W: for a step in a random
    direction the change of sum(y * dy) is the gradient times the step, up to the roundings of
    the two bf16 outputs."""
    torch, units, weight, off, d_off, x, w, dy, dev = setup(3, low_cost=False)
    rng = np.random.default_rng(30)
    xt = dev(x).requires_grad_()
    y0 = units.linear("m", xt, d_off)
    y0.backward(dev(dy))
    y0 = y0.detach().double()
    dyt = dev(dy).double()
    dyt[off[-1]:] = 0
    for which, grad in (("x", xt.grad), ("w", units.grads["m"])):
        base = xt.detach() if which == "x" else weight.detach()
        step = X.bf16(rng.standard_normal(tuple(base.shape)).astype(np.float32) * 0.25)
        moved = (base.float() + torch.from_numpy(step).cuda()).to(torch.bfloat16)
        taken = moved.double() - base.double()          # the step after its rounding
        with torch.no_grad():
            if which == "x":
                y1 = units.linear("m", moved, d_off).double()
            else:
                weight.copy_(moved)
                y1 = units.linear("m", xt.detach(), d_off).double()
        change = float(((y1 - y0) * dyt).sum())
        want = float((grad.double() * taken).sum())
        # independent roundings: within 2^-8 of each output, six deviations of their sum
        noise = 2.0 ** -8 * float(((y1.abs() + y0.abs()) * dyt.abs()).square().sum().sqrt())
        slack = 6 * noise + 2.0 ** -8 * float((grad.double() * taken).abs().square().sum().sqrt())
        assert abs(change - want) <= slack, (which, change, want, slack)
    units.close()


def test_refusals():
    torch, units, weight, off, d_off, x, w, dy, dev = setup(4)
    from paper_2606_00539_amd import torch_ops as ops
    from paper_2606_00539_amd.torch_experts import ExpertUnits

    with pytest.raises(RuntimeError, match="no gradient"):
        units.step(1.1, 1.5)
    with pytest.raises(KeyError):
        units.linear("other", dev(x), d_off)
    for bad in (weight.float(), weight[0], weight.transpose(1, 2), weight.cpu()):
        with pytest.raises(TypeError):
            ExpertUnits([("m", bad)])
    with pytest.raises(ValueError):
        ExpertUnits([("m", torch.zeros(2, 12, 16, dtype=torch.bfloat16, device="cuda"))])
    with pytest.raises(ValueError):
        ExpertUnits([])
    with pytest.raises(TypeError):
        ExpertUnits([("m", weight)], grad_dtype=torch.float16)
    xt, wt = dev(x), weight.detach()
    for bad in (lambda: ops.grouped_linear(xt.float(), wt, d_off),
                lambda: ops.grouped_linear(xt, wt, d_off.long()),
                lambda: ops.grouped_linear(xt, wt, d_off[:-1]),
                lambda: ops.grouped_linear(xt, wt, d_off.cpu()),
                lambda: ops.grouped_linear(xt, wt),
                lambda: ops.grouped_linear(xt[:, :64], wt, d_off),
                lambda: ops.grouped_linear(xt.t(), wt, d_off),
                lambda: ops.grouped_linear(xt, wt, d_off, mask=units.mask(0)),
                lambda: ops.grouped_linear(xt, wt, d_off, mask=units.mask(0)[:2], out=xt),
                lambda: ops.grouped_linear(xt, wt, d_off, out=xt),
                lambda: ops.grouped_wgrad(dev(dy), xt[1:], d_off),
                lambda: ops.grouped_wgrad(dev(dy), xt, d_off, accumulate=True),
                lambda: ops.grouped_wgrad(dev(dy), xt, d_off, dtype=torch.float16),
                lambda: ops.grouped_wgrad(dev(dy), xt, d_off, dw=wt[:2]),
                lambda: ops.grouped_wgrad(dev(dy), xt, d_off, partials=units.partials[:3]),
                lambda: ops.quantize_rows(xt.half()),
                lambda: ops.quantized_linear(xt, wt, units.codes[0][1], d_off),
                lambda: ops.quantized_linear(xt, units.codes[0][0], units.codes[0][1][0], d_off),
                lambda: ops.quantized_linear(xt, *units.codes[0], d_off, x_scale=xt[:, 0]),
                lambda: ops.orthogonalize(xt.t()), lambda: ops.orthogonalize(xt.half()),
                lambda: ops.orthogonalize(xt, out=xt.float())):
        with pytest.raises((TypeError, ValueError)):
            bad()
    from paper_2606_00539_amd import GnmrError

    for bad in (lambda: ops.grouped_linear(xt[:, 4:68], wt[:, :, :64].contiguous(), d_off),
                lambda: ops.orthogonalize(xt, steps=0),
                lambda: ops.orthogonalize(xt, eps=-1.0)):
        with pytest.raises(GnmrError):
            bad()
    units.close()


def test_update_is_the_orthogonalised_momentum():
    torch, units, weight, off, d_off, x, w, dy, dev = setup(5, counts=(40, 20, 77, 3))
    from paper_2606_00539_amd.torch_experts import OrthogonalMomentum

    opt = OrthogonalMomentum(units, lr=0.05, momentum=0.5)
    m = 0.0
    for k in range(2):
        before = weight.detach().float().cpu().numpy()
        units.linear("m", dev(np.roll(x, k, axis=0)), d_off).backward(dev(dy))
        g = units.grads["m"].double().cpu().numpy()
        opt.step()
        m = 0.5 * m + g
        want = np.stack([X.orthogonalize(a, 5, (3.4445, -4.7750, 2.0315), 1e-7,
                                         (136 / 72) ** 0.5) for a in m])
        got = before - weight.detach().float().cpu().numpy()
        # one rounding of the weight to bf16 and the update's own error (K8's test)
        slack = np.linalg.norm(2.0 ** -8 * (np.abs(before) + 0.1)) + 0.05 * 0.01 * np.linalg.norm(want)
        assert np.linalg.norm(got - 0.05 * want) <= slack
        codes, scale = units.codes[0]
        c, s = X.row_codes(weight.detach().float().cpu().numpy().reshape(-1, 72))
        assert np.array_equal(codes.cpu().numpy().reshape(-1, 72), c)
        assert np.array_equal(scale.cpu().numpy().reshape(-1), s)
        units._filled = [False]
    units.close()


def test_example_learns_and_recovers():
    require_gpu()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import moe_step

    losses, sets = moe_step.train(steps=40, seed=1, log=None)
    assert np.isfinite(losses).all()
    assert min(losses[-4:]) < 0.6 * losses[0]
    assert all(len(s) <= 3 for s in sets)
    assert any(u.endswith(".0") for u in sets[19])       # the step with the noisy expert
