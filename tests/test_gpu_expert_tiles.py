"""The grouped products and the orthogonalisation in each kernel that the rules choose
(expert_tiles.py), with a mask over uneven experts, rows of nobody holding NaN and sizes that end
inside a step or a tile, against the formulas in float64 on the device.  Tolerances as in
test_gpu_experts.py."""
import numpy as np
import pytest

import expert_tiles as T
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def ops():
    from paper_2606_00539_amd import torch_ops

    return require_gpu(), torch_ops


def close64(got, want, mag, K, rounded=True):
    slack = (K + 1) * 2.0 ** -23 * mag + (2.0 ** -8 * want.abs() if rounded else 0)
    assert bool(((got.double() - want).abs() <= slack).all())


@pytest.mark.parametrize("name", T.ROWS)
@pytest.mark.parametrize("which", ["linear", "dgrad", "quantized"])
def test_rows(which, name):
    torch, t = ops()
    K, N, counts, pad, _ = T.ROWS[name]
    _, rows, groups, o, i = T.shape(which, name)
    print(which, name, rows, groups, o, i, flush=True)
    g = torch.Generator(device="cuda").manual_seed(31)
    off = [0, rows] if counts is None else np.concatenate([[0], np.cumsum(counts)]).tolist()
    E = len(off) - 1
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.bfloat16)
    x, w = rand(rows, K), rand(E, o, i) * K ** -0.5
    x[off[-1]:] = float("nan")
    d_off = None if counts is None else torch.tensor(off, dtype=torch.int32, device="cuda")
    mask = None
    if E > 1:
        mask = (torch.arange(E, device="cuda") % 3 != 1).to(torch.uint8)
    out = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
    if which == "quantized":
        codes, scale = t.quantize_rows(w)
        q, s = t.quantize_rows(x)
        y = t.quantized_linear(x, codes, scale, d_off, mask=mask, mask_value=1, out=out)
    else:
        f = t.grouped_linear if which == "linear" else t.grouped_dgrad
        y = f(x, w, d_off, mask=mask, mask_value=1, out=out)
    assert bool((y[off[-1]:] == 0).all())
    for e, (a, b) in enumerate(zip(off[:-1], off[1:])):
        if mask is not None and e % 3 == 1:
            assert bool((y[a:b] == 7.0).all()), e
        elif which == "quantized":    # the sums are exact in float64, the rest as the kernel does it
            total = (q[a:b].double() @ codes[e].double().t().contiguous()).float()
            want = (total * (s[a:b, None] * scale[e][None, :])).to(torch.bfloat16)
            assert bool((y[a:b] == want).all()), e
        else:
            m = (w[e].t() if which == "linear" else w[e]).double().contiguous()
            p = x[a:b].double()
            close64(y[a:b], p @ m, p.abs() @ m.abs(), K)


@pytest.mark.parametrize("name", T.WGRAD)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weight_gradients(dtype, name):
    torch, t = ops()
    o, i, counts, _ = T.WGRAD[name]
    print("wgrad", dtype, name, flush=True)
    g = torch.Generator(device="cuda").manual_seed(32)
    off = np.concatenate([[0], np.cumsum(counts)]).tolist()
    E, rows = len(counts), off[-1]
    x = torch.randn(rows, i, generator=g, device="cuda", dtype=torch.bfloat16)
    dy = torch.randn(rows, o, generator=g, device="cuda", dtype=torch.bfloat16) * 1e-3
    d_off = torch.tensor(off, dtype=torch.int32, device="cuda")
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    dw = torch.full((E, o, i), float("nan"), dtype=dt, device="cuda")
    n = -(-o // 128) * -(-i // 128)
    parts = torch.full((E, n), float("nan"), device="cuda")
    t.grouped_wgrad(dy, x, d_off, dw=dw, partials=parts)
    for accumulate in (False, True):
        old = torch.zeros_like(dw)
        if accumulate:
            old = dw.clone()
            t.grouped_wgrad(dy, x, d_off, dw=dw, partials=parts, accumulate=True)
        for e, (a, b) in enumerate(zip(off[:-1], off[1:])):
            p, r = dy[a:b].double().t().contiguous(), x[a:b].double()
            was = old[e].double()
            close64(dw[e], p @ r + was, p.abs() @ r.abs() + was.abs(), b - a + 1, dtype == "bf16")
            sq = dw[e].double().square()
            sq = torch.nn.functional.pad(sq, (0, -i % 128, 0, -o % 128))
            blocks = sq.view(-(-o // 128), 128, -(-i // 128), 128).sum((1, 3)).flatten()
            assert bool(((parts[e].double() - blocks).abs() <= 300 * 2.0 ** -24 * blocks).all()), e


@pytest.mark.parametrize("flip", [False, True])
@pytest.mark.parametrize("count,m,n,runs", T.BATCH)
def test_orthogonalize(count, m, n, runs, flip):
    torch, t = ops()
    print("orthogonalize", count, m, n, flip, flush=True)
    g = torch.Generator(device="cuda").manual_seed(33)
    x = (torch.randn(count, m, n, generator=g, device="cuda") * 1e-3).to(torch.bfloat16)
    given = x.transpose(1, 2).contiguous() if flip else x
    got = t.orthogonalize(given)
    a, b, c = 3.4445, -4.7750, 2.0315
    for k in sorted({0, count // 2, count - 1}):
        v = x[k].double()
        v = v / (v.square().sum().sqrt() + 1e-7)
        for _ in range(5):
            s = v @ v.t().contiguous()
            v = a * v + (b * s + c * (s @ s)) @ v
        y = got[k].double()
        assert float(((y.t() if flip else y) - v).norm()) <= 0.00825 * float(v.norm()), k
