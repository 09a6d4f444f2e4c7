"""ExpertUnits with forward passes on several streams and backward called from another: the
gradients, their sums of squares and the update see every one of them."""
import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def test_micro_batches_on_two_streams():
    torch = require_gpu()
    from paper_2606_00539_amd.torch_experts import ExpertUnits, OrthogonalMomentum

    g = torch.Generator(device="cuda").manual_seed(9)
    w0 = (torch.randn(4, 520, 1032, generator=g, device="cuda") / 32).to(torch.bfloat16)
    x = [torch.randn(4096, 1032, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    off = torch.tensor([0, 1000, 1001, 3000, 4096], dtype=torch.int32, device="cuda")
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]

    def run(streams):
        w = torch.nn.Parameter(w0.clone())
        units = ExpertUnits([("m", w)], max_o=2, lock_len=1, low_cost=False)
        opt = OrthogonalMomentum(units, lr=0.1)
        norms = []
        for _ in range(3):
            losses = []
            for s, v in zip(streams, x):
                s.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(s):
                    losses.append(units.linear("m", v, off).float().square().sum())
            # (the order of two additions does not change a sum)
            torch.autograd.backward(losses)
            units.step(1.1, 1.5)
            opt.step()
            norms.append(units.query()["norm"])
        torch.cuda.synchronize()
        grads = units.grads["m"].clone()
        units.close()
        return norms, grads, w.detach()

    torch.cuda.synchronize()
    here = torch.cuda.current_stream()
    want = run([here, here])
    for _ in range(3):
        got = run(sides)
        assert all((a == b).all() for a, b in zip(got[0], want[0]))
        assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
