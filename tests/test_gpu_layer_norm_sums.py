"""K10's sums over rows, dweight and dbias, where many workgroups share the rows.

Exactly: with mean 0 and 1 / deviation 1 handed over, and x of small whole numbers whose rows sum to 0,
z is x, and every product and partial sum is a whole number below 2^24 that fp32 holds, whatever the
order: each row counts once or the result differs.

On ordinary values: a column's sum passes the rows of a lane's turns (rows / workgroups at most), at most
32 rows side by side, a sixteenth of the workgroups' sums and 16 wavefronts, each an addition with an
error of at most half of u = 2^-23 of the sum of the magnitudes; a term is within 84 u (1 + |z|) |dy|
(test_gpu_layer_norm.py has that), and the result's own rounding comes last."""
import math

import numpy as np
import pytest

from gpu_util import require_gpu
from oracle import blocks as K

pytestmark = pytest.mark.gpu
U = 2.0 ** -23


def ops():
    from paper_2606_00539_amd import torch_ops

    return require_gpu(), torch_ops


def whole_numbers(rows, cols, dtype):
    """(x, dy, dweight, dbias): x[r][c] = s[r] p[c], dy[r][c] = q[r] + c % 3."""
    torch = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    c = torch.arange(cols, device="cuda")
    p = (1 - 2 * (c % 2)) * (1 + c // 2 % 3)
    if cols % 2:
        p[-1] = 0
    assert int(p.sum()) == 0
    s = torch.randint(0, 4, (rows,), generator=g, device="cuda")
    s = torch.where(s < 2, s - 2, s - 1)
    q = torch.randint(-3, 4, (rows,), generator=g, device="cuda")
    dw = p * ((s * q).sum() + c % 3 * s.sum())
    db = q.sum() + rows * (c % 3)
    assert 6 * 5 * rows < 1 << 24
    x = s.to(dtype)[:, None] * p.to(dtype)[None]
    dy = q.to(dtype)[:, None] + (c % 3).to(dtype)[None]
    return x, dy, dw, db


def check_whole_numbers(rows, cols, dtype):
    torch, t = ops()
    print("layer norm's sums", rows, cols, dtype, flush=True)
    x, dy, want_w, want_b = whole_numbers(rows, cols, dtype)
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    weight = torch.ones(cols, device="cuda")
    for dx in (True, False):
        _, dw, db = t.layer_norm_backward(dy, x, mean, rstd, weight, bias=True, input_grad=dx)
        assert torch.equal(dw.double(), want_w.double()) and torch.equal(db.double(),
                                                                         want_b.double())
        del _


# every class of widths, with rows for more than one turn and more than 256 workgroups where there are
@pytest.mark.parametrize("rows,cols", [
    (1, 24), (31, 24), (70000, 24), (70001, 2), (65537, 100), (40003, 200), (30011, 500),
    (20011, 1000), (16385, 1023), (9001, 2056), (4999, 4447), (5003, 5120), (3001, 9000),
    (2049, 16384)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_row_counts_once(rows, cols, dtype):
    torch = require_gpu()
    check_whole_numbers(rows, cols, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype])


def test_every_row_counts_once_past_32_bits():
    """4.9e9 values."""
    check_whole_numbers(300000, 16384, require_gpu().bfloat16)


@pytest.mark.parametrize("rows,cols", [(70000, 24), (40003, 200), (16385, 1023), (5003, 2056)])
@pytest.mark.parametrize("dtype,wtype", [("bf16", "f32"), ("f32", "f32"), ("bf16", "bf16")])
def test_sums_of_ordinary_values(rows, cols, dtype, wtype):
    torch, t = ops()
    from paper_2606_00539_amd import gnmr_layer_norm_backward_workspace

    print("layer norm's sums", rows, cols, dtype, wtype, flush=True)
    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    g = torch.Generator(device="cuda").manual_seed(17)
    x = torch.randn(rows, cols, generator=g, device="cuda")
    # (sums that do not cancel: a mean, and a part along z)
    dy = 1e-2 * (torch.randn(rows, cols, generator=g, device="cuda") + 2.0 + x)
    x = (x + 0.5) * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))
    w = (1 + 0.3 * torch.randn(cols, generator=g, device="cuda")).to(types[wtype])
    x, dy = x.to(types[dtype]), dy.to(types[dtype])
    _, mean, rstd = t.layer_norm(x, w)
    _, dw, db = t.layer_norm_backward(dy, x, mean, rstd, w, bias=True)

    xs, ds = x.double().cpu().numpy(), dy.double().cpu().numpy()
    _, want_w, want_b = K.layer_norm_backward(ds, xs, w.double().cpu().numpy(), 1e-5)
    _, m, r = K.layer_norm(xs, None, None, 1e-5)
    z = np.abs((xs - m[:, None]) * r[:, None])
    workgroups = gnmr_layer_norm_backward_workspace(rows, cols) // (8 * cols)
    depth = math.ceil(rows / workgroups) + 32 + math.ceil(workgroups / 16) + 16
    assert depth < 250
    for got, want, terms in ((dw, want_w, np.abs(ds) * (1 + z)), (db, want_b, np.abs(ds))):
        slack = (84 + depth / 2) * U * terms.sum(0) + torch.finfo(got.dtype).eps / 2 * np.abs(want)
        off = np.abs(got.double().cpu().numpy() - want)
        assert (off <= slack).all(), np.argwhere(off > slack)[:5]
        # (and the bound would see a missing workgroup)
        if wtype == "f32":
            assert (np.abs(want) > 4 * workgroups * slack).mean() > 0.9
