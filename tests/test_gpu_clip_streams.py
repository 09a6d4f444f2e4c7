"""step_clipped on a stream of its own: the update and the next backward, on torch's current one,
see the gradients that it has scaled, with no synchronisation between."""
import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def run(given, steps=3):
    """Three steps of two micro-batches; `given()` is the stream for step_clipped.  The returned
    gradients, weights and norms are copies."""
    torch = require_gpu()
    from paper_2606_00539_amd.torch_experts import ExpertUnits, OrthogonalMomentum

    g = torch.Generator(device="cuda").manual_seed(21)
    w = torch.nn.Parameter((torch.randn(8, 1032, 1024, generator=g, device="cuda") / 32).bfloat16())
    off = torch.tensor([0, 100, 101, 300, 300, 512, 700, 900, 1024], dtype=torch.int32,
                       device="cuda")
    x = [torch.randn(1024, 1024, generator=g, device="cuda").bfloat16() for _ in range(2)]
    units = ExpertUnits([("m", w)], max_o=2, lock_len=1, low_cost=False)
    opt = OrthogonalMomentum(units, lr=0.1)
    torch.cuda.synchronize()
    norms, seen = [], []
    for _ in range(steps):
        for v in x:
            units.linear("m", v, off).float().square().sum().backward()
        stream = given()
        if hasattr(stream, "cuda_stream"):
            with torch.cuda.stream(stream):
                torch.cuda._sleep(20_000_000)       # some milliseconds late
        norms.append(units.step_clipped(1.1, 1.5, 1e-2, stream=stream))
        opt.step()
        seen.append(opt.buffers["m"].clone())
    units.linear("m", x[0], off).float().square().sum().backward()
    grads = units.grads["m"].clone()
    torch.cuda.synchronize()
    out = [*norms, *seen, grads, w.detach().clone()]
    units.close()
    return out


def test_an_update_and_the_next_backward_follow_a_clipping_elsewhere():
    torch = require_gpu()
    want = run(lambda: None)
    assert float(want[0]) > 1e-2        # (it does clip)
    side = torch.cuda.Stream()
    for how in (side, side.cuda_stream):
        got = run(lambda: how)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), how


def test_a_handle_of_the_default_stream():
    """0, also where torch's current stream is another."""
    torch = require_gpu()
    want = run(lambda: None)
    assert torch.cuda.default_stream().cuda_stream == 0
    side = torch.cuda.Stream()
    for current in (torch.cuda.default_stream(), side):
        with torch.cuda.stream(current):
            got = run(lambda: 0)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_step_elsewhere_reads_its_own_gradients_sums():
    """A late controller step on another stream, and the next backward at once."""
    torch = require_gpu()
    from paper_2606_00539_amd.torch_experts import ExpertUnits

    g = torch.Generator(device="cuda").manual_seed(22)
    w = torch.nn.Parameter((torch.randn(4, 136, 128, generator=g, device="cuda") / 11).bfloat16())
    off = torch.tensor([0, 10, 11, 40, 64], dtype=torch.int32, device="cuda")
    x = [torch.randn(64, 128, generator=g, device="cuda").bfloat16() * 2.0 ** k for k in range(4)]
    side = torch.cuda.Stream()

    def last_norms(given, n):
        """The norms of step n, with a backward behind it."""
        units = ExpertUnits([("m", w)], max_o=2, lock_len=1, low_cost=False)
        torch.cuda.synchronize()
        for v in x[:n]:
            units.linear("m", v, off).float().square().sum().backward()
            with torch.cuda.stream(given):
                torch.cuda._sleep(20_000_000)
            units.step(1.1, 1.5, stream=given)
        units.linear("m", x[n], off).float().square().sum().backward()
        out = units.query(stream=given)["norm"]
        torch.cuda.synchronize()
        units.close()
        return out
    here = torch.cuda.current_stream()
    for n in (1, 2, 3):
        assert (last_norms(side, n) == last_norms(here, n)).all()
