"""K10 (layer norm and its gradients) against plain float64 forms.

Tolerances, from the arithmetic (u = 2^-23): a lane adds at most 64 values in a row before at most
8 lanes' levels, so a sum is within 74 u of the sum of its magnitudes, the corrected mean within that of
the mean |x - mean| <= 1 / rstd, rstd within 40 u + 3 u of itself; z = (x - mean) rstd is then within
84 u (|z| + 1), y within |weight| times that and its roundings.  dx = rstd (g - m1 - z m2) with the
means m1 of g and m2 of g z: within 84 u of each of |g|, mean |g|, (1 + |z|) (mean |g| + mean |g z|) for
z's, the sums' and rstd's errors, so 256 u rstd (|g| + (1 + |z|) (mean |g| + mean |g z|)) in all.  dweight
and dbias: sums over R rows of terms that are within 84 u (1 + |z|) |dy|, (84 + R) u of the sum of those.  A
bf16 result is within 2^-8 of its value by its rounding."""
import sys

import numpy as np
import pytest

from gpu_util import require_gpu
from oracle import blocks as K

pytestmark = pytest.mark.gpu
U = 2.0 ** -23
EPS = 1e-5


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def ops():
    from paper_2606_00539_amd import torch_ops

    return require_gpu(), torch_ops


def types():
    torch = require_gpu()
    return {"bf16": torch.bfloat16, "f32": torch.float32}


def host(t):
    return t.double().cpu().numpy()


def half(t):
    """What a rounding to t's type can be off by, relative."""
    torch = require_gpu()
    return torch.finfo(t.dtype).eps / 2


def rows_in_a_buffer(t, left, right):
    """The same values as columns of a wider buffer, NaN around them."""
    torch = require_gpu()
    b = torch.full((t.shape[0] + 2, left + t.shape[1] + right), float("nan"), dtype=t.dtype,
                   device=t.device)
    v = b[1:1 + t.shape[0], left:left + t.shape[1]]
    v.copy_(t)
    return b, v


def rest_is_nan(b, v, left):
    c = b.clone()
    c[1:1 + v.shape[0], left:left + v.shape[1]] = float("nan")
    return bool(c.isnan().all())


# rows, cols, columns of the buffer to the left and right: every class of widths, its edges, odd
# ones and starts at any element
SHAPES = [(1, 1, 0, 0), (5, 2, 1, 0), (3, 7, 0, 0), (9, 8, 3, 5), (33, 63, 0, 0), (32, 64, 0, 8),
          (31, 65, 2, 3), (17, 128, 0, 0), (16, 129, 0, 1), (9, 256, 0, 0), (7, 257, 5, 0),
          (5, 511, 0, 0), (3, 512, 8, 8), (5, 513, 0, 0), (2, 1023, 0, 0), (9, 1024, 0, 0),
          (5, 1025, 1, 1), (3, 2048, 0, 0), (2, 2049, 0, 3), (3, 4096, 8, 0), (2, 4097, 0, 0),
          (1, 5120, 0, 0), (2, 5121, 7, 0), (3, 6144, 0, 0), (2, 6145, 0, 0), (2, 8192, 0, 0),
          (2, 8193, 0, 1), (2, 12288, 0, 0), (1, 12289, 0, 0), (1, 16383, 0, 0), (2, 16384, 0, 0),
          (1500, 40, 0, 0), (2700, 520, 0, 0), (600, 2056, 0, 8),
          # whole runs that do not fill their lanes, by four and by eight values
          (33, 104, 0, 0), (17, 204, 0, 4), (9, 392, 8, 0), (5, 1540, 0, 0), (1300, 2044, 4, 0),
          (3, 4456, 0, 0), (2, 11008, 0, 0), (700, 12300, 0, 1), (1603, 5120, 0, 0)]


def data(rows, cols, seed, dtype, wtype):
    torch = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    x = (normal(rows, cols) + 0.5) * torch.exp(normal(rows, 1))
    dy = normal(rows, cols) * 1e-2
    return (x.to(types()[dtype]), dy.to(types()[dtype]), (1 + 0.3 * normal(cols)).to(types()[wtype]),
            (0.2 * normal(cols)).to(types()[wtype]))


def check_forward(x, w, b, y, mean, rstd, eps=EPS, what=""):
    xs = host(x)
    ws = np.ones(x.shape[1]) if w is None else host(w)
    want, m, r = K.layer_norm(xs, None if w is None else ws, None if b is None else host(b), eps)
    z = np.abs((xs - m[:, None]) * r[:, None])
    slack = 84 * U * np.abs(ws) * (z + 1) + U * np.abs(want) + half(y) * np.abs(want) * (
        y.dtype != mean.dtype)
    got = host(y)
    assert np.isfinite(got).all() and (np.abs(got - want) <= slack).all(), (
        what, np.argwhere(np.abs(got - want) > slack)[:5])
    assert (np.abs(host(mean) - m) <= 74 * U / r + U * np.abs(m)).all(), what
    assert (np.abs(host(rstd) - r) <= 43 * U * r).all(), what


def check_backward(dy, x, w, dx, dw, db, eps=EPS, what=""):
    xs, ds = host(x), host(dy)
    ws = np.ones(x.shape[1]) if w is None else host(w)
    ex, ew, eb = K.layer_norm_backward(ds, xs, ws, eps)
    _, m, r = K.layer_norm(xs, None, None, eps)
    z = np.abs((xs - m[:, None]) * r[:, None])
    g = np.abs(ds * ws)
    slack = 256 * U * r[:, None] * (g + (1 + z) * (
        g.mean(1, keepdims=True) + (g * z).mean(1, keepdims=True)))
    if dx is not None:
        got, low = host(dx), half(dx) if dx.element_size() == 2 else 0
        assert np.isfinite(got).all() and (np.abs(got - ex) <= slack + low * np.abs(ex)).all(), (
            what, np.argwhere(np.abs(got - ex) > slack + low * np.abs(ex))[:5])
    for got, want, terms in ((dw, ew, np.abs(ds) * (1 + z)), (db, eb, np.abs(ds))):
        if got is not None:
            s = (84 + len(xs)) * U * terms.sum(0) + half(got) * np.abs(want)
            assert (np.abs(host(got) - want) <= s).all(), (what, np.argwhere(
                np.abs(host(got) - want) > s)[:5])


@pytest.mark.parametrize("dtype,wtype", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"),
                                         ("f32", "bf16")])
@pytest.mark.parametrize("rows,cols,left,right", SHAPES)
def test_forward_and_backward(rows, cols, left, right, dtype, wtype):
    torch, t = ops()
    say("layer norm", rows, cols, left, right, dtype, wtype)
    x, dy, w, b = data(rows, cols, rows + cols, dtype, wtype)
    (_, xv), (_, dv) = rows_in_a_buffer(x, left, right), rows_in_a_buffer(dy, right, left)
    buf, out = rows_in_a_buffer(torch.zeros_like(x), left, right)
    y, mean, rstd = t.layer_norm(xv, w, b, EPS, out=out)
    assert y is out and rest_is_nan(buf, out, left)
    check_forward(x, w, b, y, mean, rstd)
    y2, mean2, rstd2 = t.layer_norm(x, w, b, EPS)       # another alignment: the same bits
    assert torch.equal(y2, y) and torch.equal(mean2, mean) and torch.equal(rstd2, rstd)
    say("  backward")
    dx, dw, db = t.layer_norm_backward(dv, xv, mean, rstd, w, bias=True)
    assert dx.dtype == x.dtype and dw.dtype == db.dtype == w.dtype
    check_backward(dy, x, w, dx, dw, db)
    again = t.layer_norm_backward(dy, x, mean, rstd, w, bias=True)
    assert all(torch.equal(p, q) for p, q in zip(again, (dx, dw, db)))


def test_parts_that_are_not_wanted():
    torch, t = ops()
    say("layer norm, parts")
    x, dy, w, b = data(37, 200, 1, "f32", "f32")
    y, mean, rstd = t.layer_norm(x, None, None, EPS)
    check_forward(x, None, None, y, mean, rstd)
    check_forward(x, None, b, *t.layer_norm(x, None, b, EPS))
    check_forward(x, w, None, *t.layer_norm(x, w, None, EPS))
    full = t.layer_norm_backward(dy, x, mean, rstd, w, bias=True)
    for dx, dw, db in ((True, True, False), (True, False, True), (False, True, True),
                       (True, False, False), (False, False, False), (False, False, True)):
        got = t.layer_norm_backward(dy, x, mean, rstd, w, bias=db, input_grad=dx, weight_grad=dw)
        for on, g, f in zip((dx, dw, db), got, full):
            assert torch.equal(g, f) if on else g is None
    dx, dw, db = t.layer_norm_backward(dy, x, mean, rstd, None, bias=True)
    assert dw is None and db.dtype == torch.float32
    check_backward(dy, x, None, dx, None, db)


def test_no_rows():
    torch, t = ops()
    say("layer norm, no rows")
    x = torch.empty(0, 72, device="cuda")
    w = torch.ones(72, device="cuda")
    y, mean, rstd = t.layer_norm(x, w)
    assert y.shape == (0, 72) and mean.shape == (0,)
    dx, dw, db = t.layer_norm_backward(x, x, mean, rstd, w, bias=True)
    assert dx.shape == (0, 72) and not dw.any() and not db.any()


def test_leading_dimensions_and_strides():
    torch, t = ops()
    say("layer norm, shapes")
    x, dy, w, b = data(24, 72, 2, "f32", "f32")
    want = t.layer_norm(x, w, b)
    for shape in ((2, 3, 4, 72), (24, 1, 72)):
        y, mean, rstd = t.layer_norm(x.view(shape), w, b)
        assert y.shape == shape and mean.shape == shape[:-1]
        assert torch.equal(y.view(24, 72), want[0]) and torch.equal(mean.view(24), want[1])
        dx, _, _ = t.layer_norm_backward(dy.view(shape), x.view(shape), mean, rstd, w)
        assert dx.shape == shape
    one = t.layer_norm(x[3], w, b)
    assert one[0].shape == (72,) and one[1].shape == () and torch.equal(one[0], want[0][3])
    # rows that overlap, lie transposed, or are one row many times
    for v in (x.t().contiguous().t(), x[:1].expand(24, 72), x.flatten().as_strided((20, 72), (5, 1))):
        y, mean, rstd = t.layer_norm(v, w, b)
        c = v.contiguous()
        assert torch.equal(y, t.layer_norm(c, w, b)[0])
        d = dy[:len(v)]
        for p, q in zip(t.layer_norm_backward(d, v, mean, rstd, w, bias=True),
                        t.layer_norm_backward(d, c, mean, rstd, w, bias=True)):
            assert torch.equal(p, q)
    got = t.layer_norm_backward(dy[:1].expand(24, 72), x, want[1], want[2], w, bias=True)
    assert torch.equal(got[2], t.layer_norm_backward(dy[:1].expand(24, 72).contiguous(), x, want[1],
                                                     want[2], w, bias=True)[2])


@pytest.mark.parametrize("cols", [40, 700, 3000, 9000])
def test_a_mean_far_above_the_deviations(cols):
    """A mean 3,000 times the deviations: its own rounding would show in x - mean."""
    torch, t = ops()
    say("layer norm, large mean", cols)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = 3000.0 + torch.randn(6, cols, generator=g, device="cuda")
    dy = torch.randn(6, cols, generator=g, device="cuda")
    w = 1 + 0.1 * torch.randn(cols, generator=g, device="cuda")
    y, mean, rstd = t.layer_norm(x, w, None)
    check_forward(x, w, None, y, mean, rstd)
    dx, dw, db = t.layer_norm_backward(dy, x, mean, rstd, w, bias=True)
    check_backward(dy, x, w, dx, dw, db)


def test_values_that_are_not_finite_stay_in_their_rows():
    torch, t = ops()
    say("layer norm, non-finite")
    for cols in (40, 300, 3000):
        x, dy, w, b = data(9, cols, 4, "f32", "f32")
        want = t.layer_norm(x, w, b)
        bad = x.clone()
        bad[2, cols - 1], bad[5, 0], bad[7, 3] = float("nan"), float("inf"), -float("inf")
        y, mean, rstd = t.layer_norm(bad, w, b)
        rest = [0, 1, 3, 4, 6, 8]
        assert torch.equal(y[rest], want[0][rest]) and torch.equal(rstd[rest], want[2][rest])
        for r in (2, 5, 7):
            assert y[r].isnan().all() and rstd[r].isnan()
        dx, dw, db = t.layer_norm_backward(dy, bad, mean, rstd, w, bias=True)
        good = t.layer_norm_backward(dy, x, *want[1:], w, bias=True)
        assert torch.equal(dx[rest], good[0][rest]) and torch.equal(db, good[2])
        assert dx[[2, 5, 7]].isnan().all() and dw.isnan().all()


def test_constant_rows():
    torch, t = ops()
    say("layer norm, constant rows")
    for cols in (1, 24, 500, 2500):
        x = torch.tensor([0.0, 3.3, -700.0, 1e-30], device="cuda")[:, None].expand(4, cols)
        b = torch.arange(cols, device="cuda", dtype=torch.float32)
        check_forward(x.contiguous(), None, b, *t.layer_norm(x, None, b))


def test_many_rows():
    """More rows than workgroups can have a turn each, and offsets past 32 bits."""
    torch, t = ops()
    say("layer norm, many rows")
    x, dy, w, b = data(70000, 24, 5, "bf16", "f32")
    y, mean, rstd = t.layer_norm(x, w, b)
    check_forward(x, w, b, y, mean, rstd)
    dx, dw, db = t.layer_norm_backward(dy, x, mean, rstd, w, bias=True)
    check_backward(dy, x, w, dx, dw, db)
    del x, dy, y, dx
    rows, cols = 300000, 16384          # 4.9e9 values
    big = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    say("  filled")
    big[:3].normal_()
    big[-3:].normal_()
    big[3:-3] = big[0]
    ones = torch.ones(cols, device="cuda")
    y, mean, rstd = t.layer_norm(big, ones)
    for at in (slice(0, 3), slice(rows - 3, rows)):
        check_forward(big[at], ones, None, y[at], mean[at], rstd[at])
    say("  backward")
    dx, dw, db = t.layer_norm_backward(big, big, mean, rstd, ones, bias=True)
    for at in (slice(0, 3), slice(rows - 3, rows)):
        check_backward(big[at], big[at], ones, dx[at], None, None)
    assert torch.equal(dx[3], dx[rows - 4]) and torch.equal(y[3], y[rows - 4])


@pytest.mark.parametrize("cols", [4096, 4104, 4108, 4099, 1000, 203])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_results_past_the_caches(cols, dtype):
    """Results of more than 32 MB are written past the caches: the same as those of its parts."""
    torch, t = ops()
    rows = (17 << 20) // cols + 5
    say("layer norm past the caches", cols, dtype)
    x, _, w, b = data(rows, cols, 13, dtype, "f32")
    whole = t.layer_norm(x, w, b)
    for k in range(0, rows, rows // 5):
        at = slice(k, k + rows // 5)
        for p, q in zip(whole, t.layer_norm(x[at], w, b)):
            assert torch.equal(p[at], q)
    for at in (slice(0, 3), slice(rows - 3, rows)):
        check_forward(x[at], w, b, *(p[at] for p in whole))


def test_graph_replays_and_another_stream():
    torch, t = ops()
    say("layer norm, graph")
    x, dy, w, b = data(40, 200, 6, "bf16", "f32")

    def run():
        y, mean, rstd = t.layer_norm(x, w, b)
        return y, mean, rstd, *t.layer_norm_backward(dy, x, mean, rstd, w, bias=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        on_side = run()
    torch.cuda.current_stream().wait_stream(s)
    for p, q in zip(on_side, run()):
        assert torch.equal(p, q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    other = torch.cuda.CUDAGraph()      # a second one: workspaces of their own
    with torch.cuda.graph(other):
        out2 = run()
    for k in range(4):
        x.mul_(-1.5)
        dy.add_(0.01)
        torch.cuda.synchronize()
        graph.replay()
        other.replay()
        torch.cuda.synchronize()
        for p, p2, q in zip(out, out2, run()):
            assert torch.equal(p, q) and torch.equal(p2, q)


# -- the module ---------------------------------------------------------------------

@pytest.mark.parametrize("dtype,wtype", [("bf16", "f32"), ("f32", "f32"), ("bf16", "bf16")])
def test_module(dtype, wtype):
    torch, _ = ops()
    from paper_2606_00539_amd.torch_layers import LayerNorm

    say("LayerNorm module", dtype, wtype)
    x, dy, w, b = data(30, 136, 7, dtype, wtype)
    m = LayerNorm(136, dtype=types()[wtype])
    with torch.no_grad():
        m.weight.copy_(w)
        m.bias.copy_(b)
    x = x.view(5, 6, 136).requires_grad_()
    y = m(x)
    assert y.shape == x.shape and y.dtype == x.dtype
    y.backward(dy.view(5, 6, 136))
    check_backward(dy, x.detach().view(30, 136), w, x.grad.view(30, 136), m.weight.grad, m.bias.grad)
    # accumulating as autograd does; a gradient of any strides (a sum's is expanded)
    m.zero_grad()
    (m(x).sum() + m(x).sum()).backward()
    check_backward(torch.full_like(dy, 1.0), x.detach().view(30, 136), w, None,
                   m.weight.grad / 2, m.bias.grad / 2)
    with torch.no_grad():
        assert not m(x).requires_grad
    nobias = LayerNorm(136, bias=False, dtype=types()[wtype])
    assert nobias.bias is None and [n for n, _ in nobias.named_parameters()] == ["weight"]
    nobias(x).sum().backward()


def test_module_in_a_graph():
    """Forward and backward captured after a warm-up on another stream; weights' gradients and all."""
    torch, _ = ops()
    from paper_2606_00539_amd.torch_layers import LayerNorm

    say("LayerNorm module, graph")
    x, dy, w, b = data(30, 136, 12, "bf16", "f32")
    m = LayerNorm(136)
    with torch.no_grad():
        m.weight.copy_(w)
        m.bias.copy_(b)
    xt = x.clone().requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m(xt).backward(dy)
    torch.cuda.current_stream().wait_stream(side)
    xt.grad = m.weight.grad = m.bias.grad = None
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = m(xt)
        y.backward(dy)
    from paper_2606_00539_amd import torch_ops as t
    for k in range(4):
        with torch.no_grad():
            xt.mul_(-1.25)
        dy.add_(0.25)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, mean, rstd = t.layer_norm(xt.detach(), w, b)
        grads = t.layer_norm_backward(dy, xt.detach(), mean, rstd, w, bias=True)
        for p, q in zip((y, xt.grad, m.weight.grad, m.bias.grad), (want, *grads)):
            assert torch.equal(p, q), k


def test_module_gradients_against_differences():
    torch, _ = ops()
    from paper_2606_00539_amd.torch_layers import layer_norm

    say("layer norm, differences")
    x, dy, w, b = data(3, 24, 8, "f32", "f32")
    leaves = [v.clone().requires_grad_() for v in (x, w, b)]
    layer_norm(*leaves).backward(dy)
    h = 2.0 ** -6
    for k, leaf in enumerate(leaves):
        v = [u.detach().clone() for u in leaves]
        for i in ((0, 0), (1, 7), (2, 23)) if k == 0 else ((0,), (11,)):
            at = v[k][i].item()
            v[k][i] = at + h
            up = (layer_norm(*v).double() * dy).sum()
            v[k][i] = at - h
            down = (layer_norm(*v).double() * dy).sum()
            v[k][i] = at
            # y is within 100 u of its values (|y| below 4 here); the third derivative adds h^2
            slack = 2 * 24 * 100 * U * 4 * float(dy.abs().max()) / h + 20 * h * h * float(
                dy.abs().max()) * 24
            assert abs(float(leaf.grad[i]) - float((up - down) / (2 * h))) < slack


def test_second_derivatives_and_other_types_are_refused():
    torch, t = ops()
    from paper_2606_00539_amd.torch_layers import LayerNorm, layer_norm

    x = torch.randn(3, 24, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(layer_norm(x).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
    y = x.detach()
    w = torch.ones(24, device="cuda")
    m = torch.zeros(3, device="cuda")
    for kind, f in ((TypeError, lambda: layer_norm(y.half())),
                    (TypeError, lambda: layer_norm(y, w[:23])),
                    (TypeError, lambda: layer_norm(y, w.half())),
                    (TypeError, lambda: layer_norm(y, w, w.bfloat16())),
                    (TypeError, lambda: layer_norm(y, w.cpu())),
                    (TypeError, lambda: layer_norm(y, torch.ones(48, device="cuda")[::2])),
                    (TypeError, lambda: t.layer_norm(y, out=y.bfloat16())),
                    (TypeError, lambda: t.layer_norm(y, out=torch.empty(24, 3, device="cuda").t())),
                    (RuntimeError, lambda: t.layer_norm(y, out=y)),
                    (RuntimeError, lambda: layer_norm(y, eps=-1.0)),
                    (RuntimeError, lambda: layer_norm(torch.zeros(2, 16385, device="cuda"))),
                    (ValueError, lambda: t.layer_norm_backward(y[:2], y, m, m)),
                    (TypeError, lambda: t.layer_norm_backward(y.bfloat16(), y, m, m)),
                    (TypeError, lambda: t.layer_norm_backward(y, y, m[:2], m)),
                    (TypeError, lambda: t.layer_norm_backward(y, y, m, m.double())),
                    (TypeError, lambda: LayerNorm(24)(y.half()))):
        with pytest.raises(kind):
            f()
