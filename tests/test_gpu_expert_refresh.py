"""ExpertUnits.refresh() writes the INT8 codes where they lie: a captured forward pass and work
under way on another stream go on reading the memory that they know."""
import numpy as np
import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def make(torch):
    from paper_2606_00539_amd.torch_experts import ExpertUnits

    g = torch.Generator(device="cuda").manual_seed(5)
    w = torch.nn.Parameter((torch.randn(4, 136, 72, generator=g, device="cuda") / 8).to(
        torch.bfloat16))
    x = torch.randn(60, 72, generator=g, device="cuda").to(torch.bfloat16)
    off = torch.tensor([0, 20, 20, 41, 58], dtype=torch.int32, device="cuda")
    return ExpertUnits([("m", w)], max_o=2, lock_len=1), w, x, off


def test_a_captured_forward_follows_the_weights():
    torch = require_gpu()
    units, w, x, off = make(torch)
    where = [t.data_ptr() for t in units.codes[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.no_grad(), torch.cuda.stream(side):
        units.linear("m", x, off)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            y = units.linear("m", x, off)
    seen = []
    for k in range(4):
        with torch.no_grad():
            w.mul_(-1.5)
            units.refresh()
        assert [t.data_ptr() for t in units.codes[0]] == where
        other = torch.full((4 * 136 * 72,), 77, dtype=torch.int8, device="cuda")
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = units.linear("m", x, off).detach()
        assert torch.equal(y.view(torch.int16), want.view(torch.int16)), k
        seen.append(y.float().cpu().numpy().copy())
        del other
    assert all((a[:58] != b[:58]).any() for a, b in zip(seen, seen[1:]))
    units.close()


def test_codes_go_where_they_are_told():
    torch = require_gpu()
    from paper_2606_00539_amd import torch_ops as ops

    x = torch.randn(3, 5, 24, device="cuda")
    want = ops.quantize_rows(x)
    out = (torch.empty_like(want[0]).fill_(99), torch.full_like(want[1], 7.0))
    got = ops.quantize_rows(x, out=out)
    assert got[0] is out[0] and got[1] is out[1]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    c, s = out
    for bad in ((c.short(), s), (c[:2], s), (c, s.double()), (c, s[:2]), (c.cpu(), s), (c, s.cpu()),
                (c.transpose(0, 1), s), (c, torch.empty(3, 10, device="cuda")[:, ::2])):
        with pytest.raises((TypeError, ValueError)):
            ops.quantize_rows(x, out=bad)
