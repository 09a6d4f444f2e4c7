"""A training step of ExpertUnits captured in a graph after a warm-up on another stream."""
import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("warm_up", ["side stream", "default stream", "earlier capture"])
def test_forward_and_backward_captured_after_a_warm_up(warm_up):
    torch = require_gpu()
    from paper_2606_00539_amd.torch_experts import ExpertUnits, OrthogonalMomentum

    g = torch.Generator(device="cuda").manual_seed(15)
    w0 = (torch.randn(4, 136, 72, generator=g, device="cuda") / 8).to(torch.bfloat16)
    off = torch.tensor([0, 20, 20, 41, 58], dtype=torch.int32, device="cuda")
    xs = [torch.randn(60, 72, generator=g, device="cuda").to(torch.bfloat16) for _ in range(5)]
    dys = [torch.randn(60, 136, generator=g, device="cuda").to(torch.bfloat16) for _ in range(5)]

    def make():
        units = ExpertUnits([("m", torch.nn.Parameter(w0.clone()))], max_o=2, lock_len=1)
        return units, OrthogonalMomentum(units, lr=0.1)

    units, opt = make()
    want = []
    for x, dy in zip(xs, dys):
        units.linear("m", x, off).backward(dy)
        opt.step()
        units.zero_grad()
        want.append((units.grads["m"].clone(), units.weights[0].detach().clone()))
    units.close()

    units, opt = make()
    x, dy = xs[0].clone(), dys[0].clone()
    side = torch.cuda.Stream() if warm_up != "default stream" else torch.cuda.current_stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        units.linear("m", x, off).backward(dy)
    torch.cuda.current_stream().wait_stream(side)
    units.zero_grad()
    if warm_up == "earlier capture":
        torch.cuda.synchronize()
        earlier = torch.cuda.CUDAGraph()
        with torch.cuda.graph(earlier, stream=side):
            units.linear("m", x, off).backward(dy)
        units.zero_grad()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                       # on a stream of its own
        units.linear("m", x, off).backward(dy)
    for k in range(5):
        x.copy_(xs[k])
        dy.copy_(dys[k])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(units.grads["m"], want[k][0]), k
        opt.step()
        assert torch.equal(units.weights[0].detach(), want[k][1]), k
    units.close()
