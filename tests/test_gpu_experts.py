"""K6, K7 and K8 (products grouped by expert, the INT8 low-cost path, the
orthogonalised update) against plain float64 forms, at the sizes, loads, strides and
values where they can go wrong.

Tolerances, from the arithmetic: a bf16 result is within 2^-8 of its value by its one
rounding; an fp32 sum of K products in any order within (K + 1) 2^-23 of the sum of
their magnitudes (2^-23 a step: the matrix cores need not round to nearest); INT8
results follow fp32 operations that are exact or correctly rounded, so they have
equal bits; a sum of at most 16,384 squares, of which a lane adds at most 256 in a row
before its wavefront's and workgroup's lanes are added, within 300 * 2^-24."""
import sys

import numpy as np
import pytest

from gpu_util import require_gpu
from oracle import experts as X

pytestmark = pytest.mark.gpu
COEF = (3.4445, -4.7750, 2.0315)


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
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32).cpu().numpy()


class Wide:
    """A bf16 matrix as a slice of a buffer, NaN all around it."""

    def __init__(self, torch, values, extra):
        r, c = values.shape
        self.buf = torch.full((r + 2, c + 2 * extra), float("nan"), dtype=torch.bfloat16,
                              device="cuda")
        self.t = self.buf[1:r + 1, extra:extra + c] if extra else self.buf[1:r + 1]
        self.t.copy_(torch.from_numpy(values))

    def untouched(self):
        """The rest of the buffer is still NaN."""
        rest = self.buf.clone()
        r, c = self.t.shape
        off = (self.buf.shape[1] - c) // 2
        rest[1:r + 1, off:off + c] = float("nan")
        return bool(rest.isnan().all())


# experts' loads, rows of nobody, in, out, extra columns around the slices
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
    "63 experts": ([2] * 63, 0, 48, 56, 0),
    "few rows, wide": ([3, 0, 2, 9, 1, 17], 0, 2048, 1408, 0),
    "long": ([700, 40, 1000], 0, 520, 392, 0),
}


def load(torch, name, seed):
    counts, pad, i, o, extra = LOADS[name]
    rng = np.random.default_rng(seed)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rows = int(off[-1]) + pad
    x = X.bf16(rng.standard_normal((rows, i)).astype(np.float32) * np.exp(
        rng.standard_normal((rows, 1))).astype(np.float32))
    dy = X.bf16(rng.standard_normal((rows, o)).astype(np.float32) * 1e-3)
    w = X.bf16(rng.standard_normal((len(counts), o, i)).astype(np.float32) / np.sqrt(i))
    for m in (x, dy):
        m[off[-1]:] = np.nan                # rows of nobody may hold anything
    return off, x, dy, w, extra, torch.from_numpy(off).cuda()


def owned(off, m):
    m = m.copy()
    m[off[-1]:] = 0
    return m


def check_bf16(got, want, mag, K, what):
    bad = np.abs(got - want) > 2.0 ** -8 * np.abs(want) + (K + 1) * 2.0 ** -23 * mag
    assert not bad.any() and np.isfinite(got).all(), (what, np.argwhere(bad)[:5])


@pytest.mark.parametrize("name", LOADS)
@pytest.mark.parametrize("which", ["linear", "dgrad"])
def test_grouped_rows(which, name):
    torch, t = ops()
    say("grouped", which, name)
    off, x, dy, w, extra, d_off = load(torch, name, 1)
    src = x if which == "linear" else dy
    K, N = (w.shape[2], w.shape[1]) if which == "linear" else (w.shape[1], w.shape[2])
    a = Wide(torch, src, extra)
    out = Wide(torch, np.full((len(src), N), 7.0, np.float32), extra)
    wt = torch.from_numpy(w).to(torch.bfloat16).cuda()
    f = t.grouped_linear if which == "linear" else t.grouped_dgrad
    got = f(a.t, wt, d_off, out=out.t)
    assert got is out.t and out.untouched()
    want, mag = X.grouped_rows(owned(off, src), w.transpose(0, 2, 1) if which == "linear" else w,
                               off)
    check_bf16(host(got), want, mag, K, (which, name))
    # the same without a given output, twice: equal bits
    again = f(a.t, wt, d_off)
    assert np.array_equal(bits(again), bits(got))


@pytest.mark.parametrize("name", LOADS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_grouped_wgrad(dtype, name):
    torch, t = ops()
    say("grouped wgrad", dtype, name)
    off, x, dy, w, extra, d_off = load(torch, name, 2)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    a, b = Wide(torch, dy, extra), Wide(torch, x, extra)
    dw, parts = t.grouped_wgrad(a.t, b.t, d_off, dtype=dt)
    want, mag = X.grouped_wgrad(dy, x, off)
    K = max(np.diff(off))
    slack = (K + 1) * 2.0 ** -23 * mag + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
    assert (np.abs(host(dw) - want) <= slack).all()
    np.testing.assert_allclose(parts.cpu().numpy(), X.block_sumsq(host(dw)), rtol=300 * 2.0 ** -24)
    # accumulating: the stored value is added in fp32, then rounded
    old = host(dw)
    dw2, parts2 = t.grouped_wgrad(a.t, b.t, d_off, dw=dw, accumulate=True, partials=parts)
    assert dw2 is dw and parts2 is parts
    total = old + want
    slack = (K + 2) * 2.0 ** -23 * (mag + np.abs(old)) + (
        2.0 ** -8 * np.abs(total) if dtype == "bf16" else 0)
    assert (np.abs(host(dw) - total) <= slack).all()
    np.testing.assert_allclose(parts.cpu().numpy(), X.block_sumsq(host(dw)), rtol=300 * 2.0 ** -24)


def test_wgrad_blocks_feed_the_controller():
    """Norms of the experts as units, from the partials as they lie."""
    torch, t = ops()
    from paper_2606_00539_amd import Controller

    off, x, dy, w, _, d_off = load(torch, "tile edges", 3)
    E, o, i = w.shape
    _, parts = t.grouped_wgrad(torch.from_numpy(dy).to(torch.bfloat16).cuda(),
                               torch.from_numpy(x).to(torch.bfloat16).cuda(), d_off,
                               dtype=torch.float32)
    want, _ = X.grouped_wgrad(dy, x, off)
    with Controller(E, 5, 2, 2, 1e-12, np.zeros(E + 1, np.int64), [], []) as ctl:
        ctl.bind_partials(np.arange(E + 1) * parts.shape[1])
        ctl.step_from_partials(parts, 1.1, 1.5, torch.cuda.current_stream())
        got = ctl.query()["norm"]
    np.testing.assert_allclose(got, np.sqrt((want ** 2).sum((1, 2))), rtol=1e-5)


@pytest.mark.parametrize("value", [1, 0])
def test_masks_leave_the_others_alone(value):
    torch, t = ops()
    off, x, dy, w, _, d_off = load(torch, "tile edges", 4)
    E, o, i = w.shape
    mask = np.array([1, 0, 0, 7, 0, 1], np.uint8)          # any nonzero is 1
    on = (mask != 0) == bool(value)
    d_mask = torch.from_numpy(mask).cuda()
    xt, dyt, wt = (torch.from_numpy(m).to(torch.bfloat16).cuda() for m in (x, dy, w))
    rows_on = np.zeros(len(x), bool)
    for e in range(E):
        rows_on[off[e]:off[e + 1]] = on[e]
    rows_on[off[-1]:] = True                               # rows of nobody are always zeroed
    q, sw = t.quantize_rows(wt)
    for f in (lambda m, y: t.grouped_linear(xt, wt, d_off, mask=m, mask_value=value, out=y),
              lambda m, y: t.quantized_linear(xt, q, sw, d_off, mask=m, mask_value=value, out=y)):
        full = f(None, None)
        y = torch.full((len(x), o), 7.0, dtype=torch.bfloat16, device="cuda")
        f(d_mask, y)
        assert np.array_equal(bits(y)[rows_on], bits(full)[rows_on])
        assert (host(y)[~rows_on] == 7.0).all()
    full = t.grouped_dgrad(dyt, wt, d_off)
    dx = torch.full((len(x), i), 7.0, dtype=torch.bfloat16, device="cuda")
    t.grouped_dgrad(dyt, wt, d_off, mask=d_mask.bool(), mask_value=value, out=dx)
    assert np.array_equal(bits(dx)[rows_on], bits(full)[rows_on])
    assert (host(dx)[~rows_on] == 7.0).all()
    dw0, p0 = t.grouped_wgrad(dyt, xt, d_off)
    dw, p = torch.full_like(dw0, 7.0), torch.full_like(p0, 7.0)
    t.grouped_wgrad(dyt, xt, d_off, mask=d_mask, mask_value=value, dw=dw, partials=p)
    assert np.array_equal(bits(dw)[on], bits(dw0)[on]) and (host(dw)[~on] == 7.0).all()
    assert np.array_equal(bits(p)[on], bits(p0)[on]) and (host(p)[~on] == 7.0).all()


def test_nonfinite_values_stay_with_their_rows_and_experts():
    torch, t = ops()
    off, x, dy, w, _, d_off = load(torch, "tile edges", 5)
    x[3, 100], x[200, 0] = np.nan, np.inf
    w[3, 17, 5] = np.nan
    xt, dyt, wt = (torch.from_numpy(m).to(torch.bfloat16).cuda() for m in (x, dy, w))
    y = host(t.grouped_linear(xt, wt, d_off))
    bad = np.zeros_like(y, bool)
    bad[[3, 200]] = True
    bad[off[3]:off[4], 17] = True
    assert (~np.isfinite(y) == bad).all()
    y = host(t.quantized_linear(xt, *t.quantize_rows(wt), d_off))
    assert (~np.isfinite(y) == bad).all()
    dw = host(t.grouped_wgrad(dyt, xt, d_off)[0])
    bad = np.zeros_like(dw, bool)
    bad[0, :, 100] = bad[1, :, 0] = True
    assert (~np.isfinite(dw) == bad).all()


def test_without_offsets_one_expert_has_all_rows():
    torch, t = ops()
    off, x, dy, w, _, _ = load(torch, "one expert, all its rows", 6)
    d_off = torch.from_numpy(off).cuda()
    xt, dyt, wt = (torch.from_numpy(m).to(torch.bfloat16).cuda() for m in (x, dy, w))
    assert np.array_equal(bits(t.grouped_linear(xt, wt)), bits(t.grouped_linear(xt, wt, d_off)))
    assert np.array_equal(bits(t.grouped_dgrad(dyt, wt)), bits(t.grouped_dgrad(dyt, wt, d_off)))
    assert np.array_equal(bits(t.grouped_wgrad(dyt, xt)[0]),
                          bits(t.grouped_wgrad(dyt, xt, d_off)[0]))


# -- INT8 ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,extra", [(1, 8, 0), (5, 24, 8), (33, 1000, 0), (7, 2048, 0),
                                             (3, 13824, 16), (260, 520, 0), (2, 131064, 0)])
def test_quantize_rows(dtype, rows, cols, extra):
    torch, t = ops()
    say("quantize", dtype, rows, cols)
    rng = np.random.default_rng(rows * cols)
    x = (rng.standard_normal((rows, cols)) * np.exp(3 * rng.standard_normal((rows, 1)))).astype(
        np.float32)
    x[0, : cols // 2] = np.round(x[0, : cols // 2])
    if rows > 4:
        x[1], x[2] = 0.0, 1e-31
        x[3, cols - 1], x[4, 0] = np.nan, -np.inf
    if dtype == "bf16":
        x = X.bf16(x)
    buf = torch.full((rows, cols + 2 * extra), float("nan"), device="cuda",
                     dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    view = buf[:, extra:extra + cols] if extra else buf
    view.copy_(torch.from_numpy(x))
    codes, scale = t.quantize_rows(view)
    q, s = X.row_codes(x)
    assert np.array_equal(codes.cpu().numpy(), q)
    assert np.array_equal(scale.cpu().numpy(), s, equal_nan=True)


@pytest.mark.parametrize("rows,i,o", [(1, 8, 8), (1, 5120, 1000), (2, 136, 264), (3, 24, 40),
                                      (4, 2048, 136), (5, 1416, 520), (8, 128, 128),
                                      (16, 264, 200), (17, 256, 72), (31, 4096, 328),
                                      (33, 504, 136), (77, 1024, 1408), (128, 128, 256),
                                      (300, 776, 392), (1030, 320, 264)])
def test_quantized_linear(rows, i, o):
    torch, t = ops()
    say("quantized linear", rows, i, o)
    rng = np.random.default_rng(rows + i + o)
    x = X.bf16(rng.standard_normal((rows, i)).astype(np.float32))
    w = rng.standard_normal((o, i)).astype(np.float32)
    if rows > 1:
        x[0] = 0.0
    codes, scale = t.quantize_rows(torch.from_numpy(w).cuda())
    q, sx = X.row_codes(x)
    c, sw = X.row_codes(w)
    assert np.array_equal(codes.cpu().numpy(), c) and np.array_equal(scale.cpu().numpy(), sw)
    want = X.bf16(X.quantized_linear(q, sx, c[None], sw[None], [0, rows]))
    wide = Wide(torch, x, 8)
    out = Wide(torch, np.zeros((rows, o), np.float32), 16)
    y = t.quantized_linear(wide.t, codes, scale, out=out.t)
    assert np.array_equal(host(y), want) and out.untouched()
    xq, xs = t.quantize_rows(wide.t)
    assert np.array_equal(host(t.quantized_linear(xq, codes, scale, x_scale=xs)), want)


@pytest.mark.parametrize("name", LOADS)
def test_quantized_linear_by_expert(name):
    torch, t = ops()
    say("quantized by expert", name)
    off, x, _, w, extra, d_off = load(torch, name, 7)
    a = Wide(torch, x, extra)
    codes, scale = t.quantize_rows(torch.from_numpy(w).to(torch.bfloat16).cuda())
    q, sx = X.row_codes(owned(off, x))
    flat, sw = X.row_codes(w.reshape(-1, w.shape[2]))
    want = X.bf16(X.quantized_linear(q, sx, flat.reshape(w.shape), sw.reshape(w.shape[:2]), off))
    assert np.array_equal(host(t.quantized_linear(a.t, codes, scale, d_off)), want)


def test_quantized_linear_largest_sums():
    """All codes at +-127 and the longest K: sums next to 2^31."""
    torch, t = ops()
    i = (1 << 17) - 8
    x = torch.ones(2, i, dtype=torch.bfloat16, device="cuda")
    x[1] = -1.0
    codes = torch.full((16, i), 127, dtype=torch.int8, device="cuda")
    codes[5] = -127
    y = host(t.quantized_linear(x, codes, torch.ones(16, device="cuda")))
    v = X.bf16(np.float32(127 * 127 * i) * (np.float32(1) / np.float32(127)))
    want = np.full((2, 16), v, np.float32)
    want[:, 5] *= -1
    want[1] *= -1
    assert np.array_equal(y, want)


# -- orthogonalisation -----------------------------------------------------------------

def update(rng, m, n, strong=True):
    g = rng.standard_normal((m, n))
    if strong and min(m, n) >= 8:
        g += 3.0 * rng.standard_normal((m, 1)) * rng.standard_normal((1, n)) / np.sqrt(min(m, n))
    return (1e-3 * g).astype(np.float32)


SHAPES = [(1, 1, 1), (2, 1, 50), (1, 50, 1), (3, 8, 8), (2, 31, 33), (1, 64, 64), (2, 65, 127),
          (1, 127, 65), (2, 128, 128), (1, 129, 300), (1, 300, 129), (5, 96, 200), (1, 256, 688),
          (2, 688, 256), (1, 513, 1027)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("count,m,n", SHAPES)
def test_orthogonalize(count, m, n, dtype):
    """Five steps.  Error in the 2-norm: the last rounding adds up to 2^-8; each of the 15
    products is rounded to 2^-12, and one step multiplies what small singular values have
    got by up to 3.4445, the large ones' by less than 1: 2^-8 + 5 * 3.4445 * 3 * 2^-12 =
    0.0165 at most, of which roundings that are independent leave less than half."""
    torch, t = ops()
    say("orthogonalize", count, m, n, dtype)
    rng = np.random.default_rng(count + 7 * m + n)
    g = np.stack([update(rng, m, n) for _ in range(count)])
    if dtype == "bf16":
        g = X.bf16(g)
    gt = torch.from_numpy(g).cuda()
    if dtype == "bf16":
        gt = gt.to(torch.bfloat16)
    out = torch.full(g.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    got = host(t.orthogonalize(gt, out=out))
    for k in range(count):
        want = X.orthogonalize(g[k], 5, COEF, 1e-7)
        assert np.linalg.norm(got[k] - want) <= 0.00825 * np.linalg.norm(want), k
    if count == 1:
        assert np.array_equal(bits(t.orthogonalize(gt[0])), bits(out[0]))


@pytest.mark.parametrize("m,n", [(40, 72), (200, 72)])
def test_orthogonalize_one_step_scaled(m, n):
    """One step: three roundings of 2^-12 on values that the norm has made small, and
    the last one, element by element."""
    torch, t = ops()
    g = X.bf16(update(np.random.default_rng(9), m, n))
    want = X.orthogonalize(g, 1, (1.5, -0.5, 0.25), 1e-3, 0.2)
    got = host(t.orthogonalize(torch.from_numpy(g).to(torch.bfloat16).cuda(), steps=1,
                               coefficients=(1.5, -0.5, 0.25), eps=1e-3, scale=0.2))
    x = np.abs(g) / (np.linalg.norm(g) + 1e-3)
    p = x if m <= n else x.T
    mag = (0.75 * (p @ p.T) + 0.25 * (p @ p.T) @ (p @ p.T)) @ p
    mag = mag if m <= n else mag.T
    slack = 2.0 ** -8 * np.abs(want) + 0.2 * (4 * 2.0 ** -12 * mag + 2.0 ** -26)
    assert (np.abs(got - want) <= slack).all()


def test_orthogonalize_scale_of_the_update_does_not_matter():
    """With eps 0 a power of two leaves the same bits, tiny and huge values too."""
    torch, t = ops()
    g = torch.from_numpy(update(np.random.default_rng(10), 70, 130)).cuda()
    want = bits(t.orthogonalize(g, eps=0.0))
    for k in (-90, -30, 20, 100):
        assert np.array_equal(bits(t.orthogonalize(torch.ldexp(g, torch.tensor(k, device="cuda")),
                                                   eps=0.0)), want), k


def test_orthogonalize_zero_and_nonfinite():
    torch, t = ops()
    rng = np.random.default_rng(11)
    g = torch.from_numpy(np.stack([update(rng, 40, 90) for _ in range(4)])).cuda()
    clean = host(t.orthogonalize(g))
    g[0] = 0.0
    g[1, 3, 7] = float("nan")
    g[2, 0, 0] = float("inf")
    for eps in (1e-7, 0.0):
        got = host(t.orthogonalize(g, eps=eps))
        assert (got[0] == 0).all()
        assert np.isnan(got[1]).all() and np.isnan(got[2]).all()
    assert np.array_equal(host(t.orthogonalize(g))[3], clean[3])


# -- sizes that run in 256 tiles ---------------------------------------------------------
# (references in float64 on the device: the same formulas, one expert at a time)

def _large(torch, seed, counts, i, o, pad=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    off = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    rows = int(off[-1]) + pad
    r = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.bfloat16)
    x, dy, w = r(rows, i), r(rows, o) * 1e-3, r(len(counts), o, i) * i ** -0.5
    return off.tolist(), torch.from_numpy(off).cuda(), x, dy, w


def _close64(torch, got, want, mag, K, rounded=True):
    slack = (K + 1) * 2.0 ** -23 * mag + (2.0 ** -8 * want.abs() if rounded else 0)
    assert bool(((got.double() - want).abs() <= slack).all())


# loads whose 256 tiles leave a part of a round, and none; widths that end inside a quarter
@pytest.mark.parametrize("counts,i,o", [((3100, 17, 4800, 0, 1083), 5120, 4216),
                                        ((4096, 2048, 2048), 4096, 6144),
                                        ((9001,), 5128, 4224)])
@pytest.mark.parametrize("which", ["linear", "dgrad", "quantized"])
def test_grouped_rows_in_large_tiles(which, counts, i, o):
    torch, t = ops()
    say("large", which, counts, i, o)
    off, d_off, x, dy, w = _large(torch, 21, counts, i, o)
    if len(counts) == 1:
        x, dy, d_off = x[:off[-1]], dy[:off[-1]], None
    if which == "quantized":
        codes, scale = t.quantize_rows(w)
        q, s = t.quantize_rows(x)
        y = t.quantized_linear(x, codes, scale, d_off)
    elif which == "linear":
        y = t.grouped_linear(x, w, d_off)
    else:
        y = t.grouped_dgrad(dy, w, d_off)
    assert bool((y[off[-1]:] == 0).all())
    for e, (a, b) in enumerate(zip(off[:-1], off[1:])):
        if which == "quantized":      # the sums are exact in float64, the rest as the kernel does it
            total = (q[a:b].double() @ codes[e].double().t()).float()
            want = (total * (s[a:b, None] * scale[e][None, :])).to(torch.bfloat16)
            assert bool((y[a:b] == want).all())
            continue
        p = (x if which == "linear" else dy)[a:b].double()
        m = (w[e].t() if which == "linear" else w[e]).double().contiguous()
        _close64(torch, y[a:b], p @ m, p.abs() @ m.abs(), m.shape[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_grouped_wgrad_in_large_tiles(dtype):
    torch, t = ops()
    off, d_off, x, dy, _ = _large(torch, 22, (2500, 2047, 0, 4100), 2056, 1544)
    # four experts of at least 2,048 rows on average and 4 * 7 * 9 tiles
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    dw, parts = t.grouped_wgrad(dy, x, d_off, dtype=dt)
    old = dw.clone()
    t.grouped_wgrad(dy, x, d_off, dw=dw, accumulate=True, partials=parts)
    for e, (a, b) in enumerate(zip(off[:-1], off[1:])):
        p, r = dy[a:b].double().t().contiguous(), x[a:b].double()
        want, mag = p @ r, p.abs() @ r.abs()
        _close64(torch, old[e], want, mag, b - a, dtype == "bf16")
        _close64(torch, dw[e], want + old[e].double(), mag + old[e].double().abs(), b - a + 1,
                 dtype == "bf16")
        sq = dw[e].double().square()
        sq = torch.nn.functional.pad(sq, (0, -sq.shape[1] % 128, 0, -sq.shape[0] % 128))
        blocks = sq.view(-(-1544 // 128), 128, -(-2056 // 128), 128).sum((1, 3)).flatten()
        assert bool(((parts[e].double() - blocks).abs() <= 300 * 2.0 ** -24 * blocks).all())


@pytest.mark.parametrize("count,m,n", [(1, 4100, 6001), (1, 6001, 4100), (40, 700, 1300)])
def test_orthogonalize_in_large_tiles(count, m, n):
    """The bound of test_orthogonalize."""
    torch, t = ops()
    say("orthogonalize", count, m, n)
    g = torch.Generator(device="cuda").manual_seed(23)
    x = (torch.randn(count, m, n, generator=g, device="cuda") * 1e-3).to(torch.bfloat16)
    got = t.orthogonalize(x)
    for k in range(0, count, 13):
        v = x[k].double()
        v = v if m <= n else v.t().contiguous()
        v = v / (v.square().sum().sqrt() + 1e-7)
        for _ in range(5):
            s = v @ v.t().contiguous()
            v = COEF[0] * v + (COEF[1] * s + COEF[2] * (s @ s)) @ v
        v = v if m <= n else v.t()
        assert float((got[k].double() - v).norm()) <= 0.00825 * float(v.norm())


# -- streams and graphs ---------------------------------------------------------------

def test_another_stream_and_a_graph():
    """All calls captured together on a side stream; replays on new inputs, with eager
    work between them, give what eager calls give."""
    torch, t = ops()
    off, x, dy, w, _, d_off = load(torch, "idle experts", 12)
    x[off[-1]:], dy[off[-1]:] = 0, 0
    wt = torch.from_numpy(w).to(torch.bfloat16).cuda()
    codes, scale = t.quantize_rows(wt)
    xt = torch.from_numpy(x).to(torch.bfloat16).cuda()
    dyt = torch.from_numpy(dy).to(torch.bfloat16).cuda()

    def step():
        dw, parts = t.grouped_wgrad(dyt, xt, d_off, dtype=torch.float32)
        return (t.grouped_linear(xt, wt, d_off), t.grouped_dgrad(dyt, wt, d_off), dw, parts,
                t.quantized_linear(xt, codes, scale, d_off), t.orthogonalize(dw))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            outs = step()
    for k in range(4):
        xt.mul_(0.5 + k)
        dyt.neg_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [bits(o) for o in outs]
        want = [bits(o) for o in step()]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert np.array_equal(a, b), k


def test_device_offsets_are_read_when_the_kernels_run():
    torch, t = ops()
    off, x, _, w, _, d_off = load(torch, "tile edges", 13)
    x[off[-1]:] = 0
    xt, wt = (torch.from_numpy(m).to(torch.bfloat16).cuda() for m in (x, w))
    a = t.grouped_linear(xt, wt, d_off)
    moved = off.copy()
    moved[2:5] += 1
    d_off.copy_(torch.from_numpy(moved))
    b = t.grouped_linear(xt, wt, d_off)
    want, mag = X.grouped_rows(x, w.transpose(0, 2, 1), moved)
    check_bf16(host(b), want, mag, w.shape[2], "moved")
    assert not np.array_equal(bits(a), bits(b))
