"""K9 (gated feed-forward by expert) against plain float64 forms.

Tolerances, from the arithmetic (u = 2^-23): a bf16 result is within 2^-8 of its value by its
rounding; an fp32 sum of K products within s = (K + 1) u of the sum of their magnitudes (the matrix
cores need not round to nearest).  act: the exponential's argument is a g^k, rounded twice, so the
exponential is off by |argument| 2 u and its last bit, 1 + e and the reciprocal by a bit each, and
gelu's fitted function by 1.0e-6: act is within r = (2 |argument| + 6) u (+ 1.0e-6) of itself, its
slope within what the same relative errors make of its two terms.  |act'| < 1.13 carries the error of
the gate's sum to h."""
import sys

import numpy as np
import pytest

import block_tiles as T
from gpu_util import require_gpu
from oracle import blocks as K
from oracle import experts as X

pytestmark = pytest.mark.gpu
U = 2.0 ** -23
BF16 = 2.0 ** -8


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def ops():
    from paper_2606_00539_amd import torch_ops

    return require_gpu(), torch_ops


def host(t):
    return t.float().cpu().numpy()


def bits(t):
    torch = require_gpu()
    return t.contiguous().view(torch.int16).cpu().numpy()


class Wide:
    """A bf16 matrix as a slice of a buffer, NaN all around it."""

    def __init__(self, values, extra):
        torch = require_gpu()
        r, c = values.shape
        self.buf = torch.full((r + 2, c + 2 * extra), float("nan"), dtype=torch.bfloat16,
                              device="cuda")
        self.t = self.buf[1:r + 1, extra:extra + c] if extra else self.buf[1:r + 1]
        self.t.copy_(torch.from_numpy(values))

    def untouched(self):
        rest = self.buf.clone()
        r, c = self.t.shape
        off = (self.buf.shape[1] - c) // 2
        rest[1:r + 1, off:off + c] = float("nan")
        return bool(rest.isnan().all())


# experts' loads, rows of nobody, others, hidden, extra columns around the slices
LOADS = {
    "one row": ([1], 0, 8, 8, 0),
    "one expert, all its rows": ([300], 0, 264, 200, 8),
    "idle experts": ([0, 130, 0, 0, 1, 0], 5, 72, 136, 16),
    "nobody at all": ([0, 0, 0], 70, 64, 136, 0),
    "tile edges": ([128, 129, 127, 256, 1, 255], 1, 136, 264, 8),
    "K below a step": ([33, 31, 32], 0, 24, 40, 0),
    "K a step and a bit": ([65, 64, 63], 3, 200, 72, 0),
    "more experts than lanes": ([(7 * e) % 23 if e % 5 else 0 for e in range(150)], 9, 64, 88, 0),
    "64 experts": ([e % 3 for e in range(64)], 0, 48, 56, 8),
    "few rows, wide": ([3, 0, 2, 9, 1, 17], 0, 2048, 1408, 0),
    "long": ([700, 40, 1000], 0, 520, 392, 0),
}


def data(counts, pad, K_, H, seed):
    """(off, x, w, dy, v, pre): rows of nobody hold NaN."""
    rng = np.random.default_rng(seed)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rows, E = int(off[-1]) + pad, len(counts)
    x = X.bf16(rng.standard_normal((rows, K_)).astype(np.float32) * np.exp(
        rng.standard_normal((rows, 1))).astype(np.float32))
    w = X.bf16((rng.standard_normal((E, 2 * H, K_)) / np.sqrt(K_)).astype(np.float32))
    dy = X.bf16((1e-3 * rng.standard_normal((rows, K_))).astype(np.float32))
    v = X.bf16((rng.standard_normal((E, K_, H)) / np.sqrt(H)).astype(np.float32))
    pre = X.bf16((2.0 * rng.standard_normal((rows, 2 * H))).astype(np.float32))
    for m in (x, dy, pre):
        m[off[-1]:] = np.nan
    return off, x, w, dy, v, pre


def owned(off, m):
    m = m.copy()
    m[off[-1]:] = 0
    return m


def relative(g, kind):
    """The relative error of act at g."""
    argument = np.abs(1.45 * g) if kind == "silu" else 0.73 * g * g
    return (2 * argument + 6) * U + (0 if kind == "silu" else 1.0e-6)


def slope_error(g, kind):
    """The absolute error of act' at g, from those of its terms."""
    r = relative(g, kind)
    if kind == "silu":      # s (1 + g (1 - s)), 1 - s within s r + u
        s = 1 / (1 + np.exp(-g))
        return s * r * np.abs(1 + g * (1 - s)) + s * np.abs(g) * (s * r + U) + 3 * U * s * (
            1 + np.abs(g))
    phi, density = K.activation(np.where(g == 0, 1e-9, g), kind)[0] / np.where(
        g == 0, 1e-9, g), 0.4 * np.exp(-0.5 * g * g)
    return (phi + np.abs(g) * density) * (r + 2 * U) + U


def check_h(got, pre, mag, k, kind, what):
    g, u = np.split(pre, 2, 1)
    sg, su = np.split((k + 1) * U * mag, 2, 1)
    act = K.activation(g, kind)[0]
    h = act * u
    slack = (BF16 + 2 * U) * np.abs(h) + 1.13 * sg * (np.abs(u) + su) + np.abs(act) * su + (
        np.abs(h) * relative(g, kind)) * 1.01 + 1e-37
    bad = np.abs(got - h) > slack
    assert not bad.any() and np.isfinite(got).all(), (what, np.argwhere(bad)[:5])


def check_dgrad(got, dy, v, pre, off, kind, what):
    d, mag = X.grouped_rows(dy, v, off)
    sd = (v.shape[1] + 1) * U * mag
    g, u = np.split(pre.astype(np.float64), 2, 1)
    act, slope = K.activation(g, kind)
    dg, du = d * slope * u, d * act
    slack_g = (BF16 + 3 * U) * np.abs(dg) + np.abs(u) * (
        sd * (np.abs(slope) + 1e-5) + np.abs(d) * slope_error(g, kind)) * 1.01 + 1e-37
    slack_u = (BF16 + 3 * U) * np.abs(du) + (
        np.abs(act) * sd + np.abs(du) * relative(g, kind)) * 1.01 + 1e-37
    want = np.concatenate([dg, du], 1)
    bad = np.abs(got - want) > np.concatenate([slack_g, slack_u], 1)
    assert not bad.any() and np.isfinite(got).all(), (what, np.argwhere(bad)[:5])


def check(off, x, w, dy, v, pre, extra, kind, offsets, what):
    torch, t = ops()
    rows, H = len(x), v.shape[2]
    h, kept = Wide(np.full((rows, H), 7.0, np.float32), extra), Wide(
        np.full((rows, 2 * H), 7.0, np.float32), extra)
    a = Wide(x, extra)
    wt, vt = (torch.from_numpy(m).to(torch.bfloat16).cuda() for m in (w, v))
    out = t.gated_linear(a.t, wt, offsets, activation=kind, out=h.t, pre=kept.t)
    assert out[0] is h.t and out[1] is kept.t and h.untouched() and kept.untouched()
    _, p, mag = K.gated_linear(owned(off, x), w, off, kind)
    got = host(kept.t)
    bad = np.abs(got - p) > BF16 * np.abs(p) + (x.shape[1] + 1) * U * mag
    assert not bad.any() and np.isfinite(got).all(), (what, np.argwhere(bad)[:5])
    check_h(host(h.t), p, mag, x.shape[1], kind, what)
    # without the products, and with new ones: the same bits
    assert np.array_equal(bits(t.gated_linear(a.t, wt, offsets, activation=kind)), bits(h.t))
    again = t.gated_linear(a.t, wt, offsets, activation=kind, keep=True)
    assert np.array_equal(bits(again[0]), bits(h.t)) and np.array_equal(bits(again[1]), bits(kept.t))

    say("  gradient")
    b, c = Wide(dy, extra), Wide(pre, extra)
    dp = Wide(np.full((rows, 2 * H), 7.0, np.float32), extra)
    assert t.gated_dgrad(b.t, vt, c.t, offsets, activation=kind, out=dp.t) is dp.t
    assert dp.untouched()
    check_dgrad(host(dp.t), owned(off, dy), v, owned(off, pre), off, kind, what)
    assert np.array_equal(bits(t.gated_dgrad(b.t, vt, c.t, offsets, activation=kind)), bits(dp.t))

    say("  activation")
    h2 = Wide(np.full((rows, H), 7.0, np.float32), extra)
    assert t.gated_activation(c.t, offsets, activation=kind, out=h2.t) is h2.t and h2.untouched()
    q = owned(off, pre).astype(np.float64)
    check_h(host(h2.t), q, np.zeros_like(q), 0, kind, what)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
@pytest.mark.parametrize("name", LOADS)
def test_loads(name, kind):
    torch, _ = ops()
    say("gated", name, kind)
    counts, pad, k, H, extra = LOADS[name]
    off, *rest = data(counts, pad, k, H, 1)
    check(off, *rest, extra, kind, torch.from_numpy(off).cuda(), (name, kind))


@pytest.mark.parametrize("rows", [1, 2, 63, 129])
def test_without_offsets(rows):
    say("gated without offsets", rows)
    off, *rest = data([rows], 0, 72, 104, 2)
    check(off, *rest, 8, "silu", None, rows)


@pytest.mark.parametrize("name", T.SHAPES)
def test_every_kernel(name):
    """Random rows of the result against float64 (all of them take too long at these sizes), all
    of it against the products of the same rows one expert at a time."""
    torch, t = ops()
    say("gated", name)
    H, k, counts, pad, _ = T.SHAPES[name]
    g = torch.Generator(device="cuda").manual_seed(5)
    E = 1 if counts is None else len(counts)
    off = np.concatenate([[0], np.cumsum([pad] if counts is None else counts)]).astype(np.int32)
    rows = pad if counts is None else int(off[-1]) + pad
    d_off = None if counts is None else torch.from_numpy(off).cuda()

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(torch.bfloat16)
    x, w = normal(rows, k), normal(E, 2 * H, k, scale=k ** -0.5)
    dy, v, pre = normal(rows, k, scale=1e-3), normal(E, k, H, scale=H ** -0.5), normal(rows, 2 * H)
    for m in (x, dy, pre):
        m[off[-1]:] = float("nan")
    kind = "gelu" if "one expert" in name else "silu"
    h, kept = t.gated_linear(x, w, d_off, activation=kind, keep=True)
    say("  nothing kept")
    alone = t.gated_linear(x, w, d_off, activation=kind)
    say("  gradient")
    dp = t.gated_dgrad(dy, v, pre, d_off, activation=kind)
    assert not any(m[off[-1]:].any() for m in (h, alone, kept, dp))
    rng = np.random.default_rng(6)
    # the first and the last row of some experts, and others
    pick = sorted({int(r) for e in rng.permutation(E)[:12] if off[e + 1] > off[e]
                   for r in (off[e], off[e + 1] - 1, rng.integers(off[e], off[e + 1]))})
    of = np.searchsorted(off, pick, side="right") - 1
    for r, e in zip(pick, of):
        one = np.array([0, 1])
        xs, ws = host(x[r:r + 1]), host(w[e:e + 1])
        _, p, mag = K.gated_linear(xs, ws, one, kind)
        got = host(kept[r:r + 1])
        assert (np.abs(got - p) <= BF16 * np.abs(p) + (k + 1) * U * mag).all(), (name, r)
        check_h(host(h[r:r + 1]), p, mag, k, kind, (name, r))
        check_h(host(alone[r:r + 1]), p, mag, k, kind, (name, r))
        check_dgrad(host(dp[r:r + 1]), host(dy[r:r + 1]), host(v[e:e + 1]), host(pre[r:r + 1]), one,
                    kind, (name, r))
    # the whole, expert by expert, in fp32 on the device: far looser, but no tile is left out
    for e in range(E):
        a, b = int(off[e]), int(off[e + 1])
        if a == b:
            continue
        p = x[a:b].float() @ w[e].float().t()
        assert (kept[a:b].float() - p).norm() < 4e-3 * p.norm(), (name, e)
        z = p[:, :H]
        z = z * torch.sigmoid(z) if kind == "silu" else z * torch.special.ndtr(z)
        z = z * p[:, H:]
        assert (h[a:b].float() - z).norm() < 4e-3 * z.norm(), (name, e)
        assert (alone[a:b].float() - z).norm() < 4e-3 * z.norm(), (name, e)
        q = pre[a:b].float().requires_grad_()
        act = torch.nn.functional.silu if kind == "silu" else torch.nn.functional.gelu
        d = dy[a:b].float() @ v[e].float()
        want, = torch.autograd.grad(act(q[:, :H]) * q[:, H:], q, d)
        assert (dp[a:b].float() - want).norm() < 4e-3 * want.norm(), (name, e)


def test_masks_send_each_expert_down_one_path():
    torch, t = ops()
    say("gated masks")
    off, x, w, dy, v, pre = data([40, 0, 77, 3], 6, 72, 136, 3)
    d_off, mask = torch.from_numpy(off).cuda(), torch.tensor([1, 1, 0, 1], dtype=torch.uint8,
                                                             device="cuda")
    cuda = [torch.from_numpy(m).to(torch.bfloat16).cuda() for m in (x, w, dy, v, pre)]
    xt, wt, dyt, vt, pt = cuda
    h_all, p_all = t.gated_linear(xt, wt, d_off, keep=True)
    d_all, a_all = t.gated_dgrad(dyt, vt, pt, d_off), t.gated_activation(pt, d_off)
    mine = torch.ones(len(x), dtype=torch.bool, device="cuda")
    mine[int(off[2]):int(off[3])] = False       # (rows of nobody are written by either call)
    for value in (1, 0):
        h, p, d, a = (torch.full_like(m, 7.0) for m in (h_all, p_all, d_all, a_all))
        t.gated_linear(xt, wt, d_off, mask=mask.bool(), mask_value=value, out=h, pre=p)
        t.gated_dgrad(dyt, vt, pt, d_off, mask=mask, mask_value=value, out=d)
        t.gated_activation(pt, d_off, mask=mask, mask_value=value, out=a)
        at = mine if value else ~mine
        at = at.clone()
        at[int(off[-1]):] = True
        for got, want in ((h, h_all), (p, p_all), (d, d_all), (a, a_all)):
            assert torch.equal(got[at], want[at]) and bool((got[~at] == 7.0).all())


def test_values_that_are_not_finite_stay_in_their_rows():
    torch, t = ops()
    say("gated non-finite")
    off, x, w, dy, v, pre = data([40, 24], 0, 72, 136, 4)
    d_off = torch.from_numpy(off).cuda()
    wt, vt = (torch.from_numpy(m).to(torch.bfloat16).cuda() for m in (w, v))

    def run(x, dy, pre):
        x, dy, pre = (torch.from_numpy(m).to(torch.bfloat16).cuda() for m in (x, dy, pre))
        return (*t.gated_linear(x, wt, d_off, keep=True), t.gated_dgrad(dy, vt, pre, d_off),
                t.gated_activation(pre, d_off))
    want = run(x, dy, pre)
    x2, dy2, pre2 = x.copy(), dy.copy(), pre.copy()
    x2[7, 3], dy2[9, 5], pre2[50, 4], pre2[51, 140] = np.nan, np.inf, np.nan, np.inf
    got = run(x2, dy2, pre2)
    for k, bad in enumerate(((7,), (7,), (9, 50, 51), (50, 51))):
        rest = [r for r in range(64) if r not in bad]
        assert torch.equal(got[k][rest], want[k][rest])
        assert all(not got[k][r].isfinite().all() for r in bad)
    # single values: only their columns
    assert int((~got[3][50].isfinite()).sum()) == 1 and int((~got[3][51].isfinite()).sum()) == 1


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gates_over_their_whole_range(kind):
    """Every bf16 gate between -3e38 and 3e38, of which most have act 0 or g."""
    torch, t = ops()
    say("gated range", kind)
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    every = every[every.isfinite()]
    n = len(every) // 8 * 8
    pre = torch.stack([every[:n], torch.ones(n, dtype=torch.bfloat16)]).view(1, 2 * n).cuda()
    h = host(t.gated_activation(pre, activation=kind))[0]
    g = every[:n].double().numpy()
    with np.errstate(under="ignore"):
        want = K.activation(g, kind)[0]
    # the hardware's exponential and reciprocal are 0 below 2^-126, where s (or F) is: act = g s is then
    # off by as much as |g| 2^-126, and by half of the smallest bf16 value besides
    slack = BF16 * np.abs(want) + np.abs(want) * relative(np.clip(np.abs(g), 0, 200), kind) + (
        2.0 ** -126 * np.minimum(np.abs(g), 200) + 2.0 ** -133)
    assert (np.abs(h - want) <= slack).all(), g[np.abs(h - want) > slack][:10]


def test_graph_replays_and_another_stream():
    torch, t = ops()
    say("gated graph")
    off, x, w, dy, v, pre = data([40, 0, 77, 3], 6, 72, 136, 5)
    d_off = torch.from_numpy(off).cuda()
    x, w, dy, v, pre = (torch.from_numpy(m).to(torch.bfloat16).cuda() for m in (x, w, dy, v, pre))

    def run():
        return (*t.gated_linear(x, w, d_off, keep=True), t.gated_dgrad(dy, v, pre, d_off),
                t.gated_activation(pre, d_off))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        on_side = run()
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(on_side, run()):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for k in range(4):
        x.mul_(-0.5)
        d_off[1:3] += 1 if k % 2 == 0 else -1       # a row more or less for the first expert
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, run()):
            assert torch.equal(a, b)


def test_refusals():
    torch, t = ops()
    x = torch.zeros(4, 16, dtype=torch.bfloat16, device="cuda")
    w = torch.zeros(2, 32, 16, dtype=torch.bfloat16, device="cuda")
    off = torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda")
    mask = torch.ones(2, dtype=torch.uint8, device="cuda")
    v = torch.zeros(2, 16, 16, dtype=torch.bfloat16, device="cuda")
    pre = torch.zeros(4, 32, dtype=torch.bfloat16, device="cuda")
    h = torch.zeros(4, 16, dtype=torch.bfloat16, device="cuda")
    for kind, f in (
            (ValueError, lambda: t.gated_linear(x, w, off, activation="relu")),
            (ValueError, lambda: t.gated_linear(x, w)),
            (ValueError, lambda: t.gated_linear(x, w, off, mask=mask)),
            (ValueError, lambda: t.gated_linear(x, w, off, mask=mask, out=h, keep=True)),
            (ValueError, lambda: t.gated_linear(x, w[:, :31].contiguous(), off)),
            (ValueError, lambda: t.gated_linear(x[:, :8], w, off)),
            (ValueError, lambda: t.gated_linear(x, w, off, out=pre)),
            (ValueError, lambda: t.gated_linear(x, w, off, pre=h)),
            (TypeError, lambda: t.gated_linear(x.float(), w, off)),
            (TypeError, lambda: t.gated_linear(x, w.float(), off)),
            (TypeError, lambda: t.gated_linear(x, w, off.long())),
            (ValueError, lambda: t.gated_dgrad(x, v, h, off)),
            (ValueError, lambda: t.gated_dgrad(x[:3], v, pre, off)),
            (ValueError, lambda: t.gated_dgrad(x, v, pre, off, activation="SILU")),
            (ValueError, lambda: t.gated_dgrad(x, v, pre, off, mask=mask)),
            (ValueError, lambda: t.gated_activation(pre, off, mask=mask)),
            (ValueError, lambda: t.gated_activation(pre[:, :31], off)),
            (ValueError, lambda: t.gated_activation(pre.t(), None)),
            (RuntimeError, lambda: t.gated_linear(x, w, off, out=x)),
            (RuntimeError, lambda: t.gated_dgrad(x, v, pre, off, out=pre)),
            (RuntimeError, lambda: t.gated_linear(x, w, off, out=pre[:, :16], pre=pre))):
        with pytest.raises(kind):
            f()
