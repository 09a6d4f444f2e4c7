"""K11 (the global norm, and gradients clipped by it) against float64 forms.

Tolerances, from the arithmetic: squares of bf16 and fp32 values are exact in float64 and their sums
within n 2^-53, so norm and factor are within 1e-12 for what is tested; a scaled value is rounded
to fp32 (2^-24), and a bf16 one once more (2^-8); values below the normal range by half of the
smallest one."""
import math
import sys

import numpy as np
import pytest

from gpu_util import require_gpu
from oracle import blocks as K

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def ops():
    from paper_2606_00539_amd import torch_ops

    return require_gpu(), torch_ops


def tensors(sizes, seed, mixed=True, scale=1.0, gap=1):
    """Gradients of these sizes behind one another in a buffer of each type (so at any element),
    alternately bf16 and fp32, with NaN between them."""
    torch = require_gpu()
    g = torch.Generator(device="cuda").manual_seed(seed)
    out, bufs = [], []
    for dtype in (torch.bfloat16, torch.float32):
        mine = [n for k, n in enumerate(sizes) if not mixed or k % 2 == (dtype == torch.float32)]
        if not mixed and dtype == torch.bfloat16:
            mine = []
        buf = torch.full((sum(mine) + gap * (len(mine) + 1),), float("nan"), dtype=dtype,
                         device="cuda")
        bufs.append(buf)
    at = [gap, gap]
    for k, n in enumerate(sizes):
        f = 1 if not mixed else k % 2
        v = bufs[f][at[f]:at[f] + n]
        v.copy_(torch.randn(n, generator=g, device="cuda") * scale * math.exp(0.1 * (k % 7)))
        at[f] += n + gap
        out.append(v)
    return out, bufs


def host(t):
    return t.double().cpu().numpy()


def check_scaled(got, was, factor):
    for o, g in zip(got, was):
        if not g.numel():
            continue
        want = host(g) * factor
        low = 2.0 ** -8 if o.element_size() == 2 else 0.0
        tiny = 2.0 ** -133 if o.element_size() == 2 else 2.0 ** -149
        assert (np.abs(host(o) - want) <= (2.0 ** -24 + 1e-12 + low) * np.abs(want) + tiny).all()


SIZES = {
    "one value": [1],
    "one tensor": [100003],
    "none of some": [0, 5, 0, 0, 2047, 0],
    "edges": [2047, 2048, 2049, 7, 8, 9, 4096, 16384, 16385],
    "many": [(37 * k) % 513 for k in range(400)],
    "as many as a launch takes": [64] * 112,
    "one more": [65] * 113,
    "large": [3_000_001, 5, 20_000_000, 64],
}


@pytest.mark.parametrize("name", SIZES)
@pytest.mark.parametrize("ratio", [0.25, 4.0])
def test_in_place(name, ratio):
    torch, t = ops()
    say("clip", name, ratio)
    sizes = SIZES[name]
    gs, bufs = tensors(sizes, 1)
    was, before = [g.clone() for g in gs], [b.clone() for b in bufs]
    norm, _ = K.clip([host(g) for g in gs], [], 1.0, 0.0)
    got = t.clip_gradients(gs, ratio * norm, eps=1e-6)
    assert got.dtype == torch.float64 and got.shape == ()
    assert abs(float(got) - norm) <= 1e-12 * norm
    if ratio > 1:
        for a, b in zip(bufs, before):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    else:
        check_scaled(gs, was, ratio * norm / (norm + 1e-6))
        for a, b in zip(bufs, before):      # what lies between the gradients
            assert int(a.isnan().sum()) == int(b.isnan().sum())
        # what was clipped has the norm that was asked for
        again = float(t.clip_gradients(gs, math.inf))
        assert abs(again - ratio * norm) <= (2.0 ** -8 * norm + 1e-6) * ratio


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("ratio", [0.25, 4.0])
def test_into_other_tensors(out, ratio):
    torch, t = ops()
    say("clip into", out, ratio)
    gs, bufs = tensors(SIZES["edges"], 2)
    before = [b.clone() for b in bufs]
    dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[out]
    flat = torch.full((sum(SIZES["edges"]) + 30,), 7.0, dtype=dtype, device="cuda")
    outs, at = [], 3
    for g in gs:
        outs.append(flat[at:at + g.numel()])
        at += g.numel() + 1
    norm, factor = K.clip([host(g) for g in gs], [], 1.0, 0.0)
    norm, factor = K.clip([host(g) for g in gs], [], ratio * norm, 1e-6)
    got = t.clip_gradients(gs, ratio * norm, out=outs)
    assert abs(float(got) - norm) <= 1e-12 * norm
    check_scaled(outs, gs, factor)
    for a, b in zip(bufs, before):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert (flat[:3] == 7.0).all() and (flat[at:] == 7.0).all()


def test_norms_that_are_known():
    torch, t = ops()
    say("clip, known norms")
    gs, _ = tensors([500, 3000, 70000, 9, 2048], 3)
    norm, _ = K.clip([host(g) for g in gs], [], 1.0, 0.0)
    known = [1, 2, 4]
    norms = torch.tensor([math.sqrt(sum(float((host(gs[k]) ** 2).sum()) for k in (1, 4))),
                          float(np.linalg.norm(host(gs[2])))], dtype=torch.float64, device="cuda")
    was = [g.clone() for g in gs]
    got = t.clip_gradients(gs, 0.5 * norm, known=known, norms=norms)
    assert abs(float(got) - norm) <= 1e-12 * norm
    check_scaled(gs, was, 0.5 * norm / (norm + 1e-6))
    # all known; norms of tensors that are not given at all; more norms than a workgroup adds alone
    gs = [w.clone() for w in was]
    many = torch.full((5000,), 2.0, dtype=torch.float64, device="cuda")
    got = t.clip_gradients(gs, 10.0, known=range(5), norms=many)
    assert abs(float(got) - math.sqrt(20000.0)) <= 1e-12 * 200
    check_scaled(gs, was, 10.0 / (math.sqrt(20000.0) + 1e-6))


def test_the_whole_range_of_values():
    """Squares that fp32 has not: norms of 1e38 and of 1e-38."""
    torch, t = ops()
    say("clip, range")
    for scale in (3e37, 1e-38, 1e-41):
        gs, _ = tensors([1000, 3000], 4, mixed=False, scale=scale)
        norm, _ = K.clip([host(g) for g in gs], [], 1.0, 0.0)
        was = [g.clone() for g in gs]
        got = t.clip_gradients(gs, norm / 8, eps=0.0)
        assert abs(float(got) - norm) <= 1e-12 * norm
        check_scaled(gs, was, 0.125)


def test_values_that_are_not_finite():
    torch, t = ops()
    say("clip, non-finite")
    for bad, want in ((float("inf"), math.inf), (float("nan"), math.nan)):
        gs, _ = tensors([100, 300], 5)
        gs[1][7] = bad
        norm = float(t.clip_gradients(gs, 1.0))
        assert norm == want or (math.isnan(norm) and math.isnan(want))
        if math.isinf(want):
            assert not gs[0].any() and gs[1][7].isnan() and int(gs[1].isnan().sum()) == 1
        else:
            assert gs[0].isnan().all() and gs[1].isnan().all()
    gs, _ = tensors([100], 6)
    norms = torch.tensor([math.inf], dtype=torch.float64, device="cuda")
    assert math.isinf(float(t.clip_gradients(gs, 1.0, norms=norms))) and not gs[0].any()


def test_edges_of_the_arguments():
    torch, t = ops()
    say("clip, arguments")
    gs, _ = tensors([100, 300], 7)
    was = [g.clone() for g in gs]
    norm, _ = K.clip([host(g) for g in gs], [], 1.0, 0.0)
    assert abs(float(t.clip_gradients(gs, math.inf)) - norm) < 1e-12 * norm
    assert all(torch.equal(a, b) for a, b in zip(gs, was))
    # exactly at the bound nothing is clipped; eps counts
    assert float(t.clip_gradients(gs, float(t.clip_gradients(gs, math.inf)), eps=0.0)) > 0
    assert all(torch.equal(a, b) for a, b in zip(gs, was))
    t.clip_gradients(gs, norm, eps=norm)
    check_scaled(gs, was, 0.5)
    t.clip_gradients(gs, 0.0)
    assert not gs[0].any() and not gs[1].any()
    assert float(t.clip_gradients(gs, 0.0, eps=0.0)) == 0.0     # 0 / 0: nothing to clip
    empty = [torch.empty(0, device="cuda")]
    assert float(t.clip_gradients(empty, 1.0)) == 0.0
    signs = torch.tensor([-0.0, 0.0, -1e-45, 1.0], device="cuda")
    keep = signs.clone()
    t.clip_gradients([signs], 5.0)
    assert torch.equal(signs.view(torch.int32), keep.view(torch.int32))


def test_many_launches():
    torch, t = ops()
    say("clip, many tensors")
    buf = torch.randn(40 * 1200, device="cuda")
    gs = list(buf.view(1200, 40).unbind(0))
    was = buf.clone()
    norm = float(np.linalg.norm(host(was)))
    assert abs(float(t.clip_gradients(gs, norm / 2, eps=0.0)) - norm) <= 1e-12 * norm
    check_scaled([buf], [was], 0.5)


def test_offsets_past_32_bits():
    torch, t = ops()
    say("clip, large")
    n = (1 << 32) + 12345
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    say("  filled")
    g[-3:] = 4.0
    g[5] = 3.0
    norm = math.sqrt(3 * 16.0 + 9.0)
    assert abs(float(t.clip_gradients([g], norm / 4, eps=0.0)) - norm) < 1e-12 * norm
    assert g[-3:].tolist() == [1.0] * 3 and float(g[5]) == 0.75 and int((g != 0).sum()) == 4


def test_repeats_graphs_and_streams():
    torch, t = ops()
    say("clip, graph")
    gs, _ = tensors([5000, 70000, 3, 300000], 8)
    outs = [torch.empty_like(g) for g in gs]

    def run(to):
        return t.clip_gradients(gs, 1.0, out=to)
    first = run(outs).clone()
    want = [o.clone() for o in outs]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        second = run(outs)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(first, second) and all(torch.equal(a, b) for a, b in zip(outs, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = run(outs)
    for k in range(4):
        for g in gs:
            g.mul_(-1.25)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        other = [torch.empty_like(g) for g in gs]
        assert torch.equal(run(other), norm)
        assert all(torch.equal(a, b) for a, b in zip(outs, other))


def test_refusals():
    torch, t = ops()
    g = torch.zeros(8, 16, device="cuda")
    norms = torch.ones(2, dtype=torch.float64, device="cuda")
    for kind, f in ((TypeError, lambda: t.clip_gradients([g.half()], 1.0)),
                    (TypeError, lambda: t.clip_gradients([g.t()], 1.0)),
                    (TypeError, lambda: t.clip_gradients([g.cpu()], 1.0)),
                    (TypeError, lambda: t.clip_gradients([g], 1.0, out=[g.half()])),
                    (ValueError, lambda: t.clip_gradients([g], 1.0, out=[g.flatten().clone()])),
                    (TypeError, lambda: t.clip_gradients([g], 1.0, norms=norms.float())),
                    (TypeError, lambda: t.clip_gradients([g], 1.0, norms=norms.cpu())),
                    (ValueError, lambda: t.clip_gradients([g], 1.0, known=[1], norms=norms)),
                    (ValueError, lambda: t.clip_gradients([g], 1.0, known=[0])),
                    (RuntimeError, lambda: t.clip_gradients([g, g], 1.0)),
                    (RuntimeError, lambda: t.clip_gradients([g[:4], g[3:]], 1.0)),
                    (RuntimeError, lambda: t.clip_gradients([g[:4], g[4:]], 1.0,
                                                            out=[g[4:], g[:4]])),
                    (RuntimeError, lambda: t.clip_gradients([g], -1.0)),
                    (RuntimeError, lambda: t.clip_gradients([g], math.nan)),
                    (RuntimeError, lambda: t.clip_gradients([g], 1.0, eps=-1.0))):
        with pytest.raises(kind):
            f()
