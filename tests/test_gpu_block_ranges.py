"""The ranges that a gated block's operators are documented for, at their ends."""
import math

import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def units_of(kind, value):
    """(units, their gradients): one unit of 4096 gradients +-value (a norm of 64 value)."""
    torch = require_gpu()
    from paper_2606_00539_amd import torch_experts, torch_units

    sign = 1.0 - 2.0 * (torch.arange(4096, device="cuda") % 2)
    if kind == "TorchUnits":
        p = torch.nn.Parameter(torch.zeros(64, 64, device="cuda"))
        p.grad = (sign * value).view(64, 64)
        return torch_units.TorchUnits([("w", p)], max_o=1, lock_len=1), [p.grad]
    if kind == "FusedWgradUnits":
        m = torch.nn.Linear(64, 64, bias=False).to("cuda", torch.bfloat16)
        units = torch_units.FusedWgradUnits([("m", m)], max_o=1, lock_len=1)
        x = torch.eye(64, device="cuda").bfloat16()
        m(x).backward((sign * value).view(64, 64).bfloat16())
        return units, [m.weight.grad]
    w = torch.nn.Parameter(torch.zeros(1, 64, 64, device="cuda", dtype=torch.bfloat16))
    units = torch_experts.ExpertUnits([("m", w)], max_o=1, lock_len=1, low_cost=False)
    off = torch.tensor([0, 64], dtype=torch.int32, device="cuda")
    x = torch.eye(64, device="cuda").bfloat16()
    units.linear("m", x, off).backward((sign * value).view(64, 64).bfloat16())
    return units, list(units.grads.values())


@pytest.mark.parametrize("kind", ["TorchUnits", "FusedWgradUnits", "ExpertUnits"])
def test_step_clipped_has_the_range_of_the_controllers_norms(kind):
    torch = require_gpu()
    for power in (57, 58, -60, -76):
        print(kind, power, flush=True)
        value = 2.0 ** power
        units, gradients = units_of(kind, value)
        was = [g.clone() for g in gradients]
        other = torch.full((9,), value / 4, device="cuda")
        kept = other.clone()
        norm, own = 64.0 * value, 3.0 * value / 4
        got = float(units.step_clipped(1.1, 1.5, norm / 2, others=[other], eps=0.0))
        if power == 58:         # a unit's norm of 2^64
            assert got == math.inf and not other.any() and not any(g.any() for g in gradients)
        elif power == -76:      # its values do not count; those of `others` do
            assert got == own
            assert torch.equal(other, kept) and all(map(torch.equal, gradients, was))
        else:
            total = math.hypot(norm, own)
            assert abs(got - total) <= 1e-5 * total
            for g, w in zip([*gradients, other], [*was, kept]):
                want = w.double() * (norm / 2 / got)
                assert ((g.double() - want).abs() <= (2.0 ** -8 + 1e-6) * want.abs()).all()
        units.close()


@pytest.mark.parametrize("cols", [64, 1000, 16384])
def test_layer_norm_of_the_largest_and_smallest_deviations(cols):
    """Deviations +-2^k are powers of two in every formula: y is +-1 exactly."""
    torch = require_gpu()
    from paper_2606_00539_amd import torch_ops as t

    sign = (1.0 - 2.0 * (torch.arange(cols, device="cuda") % 2)).expand(3, cols).contiguous()
    top = (127 - math.ceil(math.log2(cols))) // 2
    for power, eps in ((top, 1e-5), (top, 0.0), (-63, 0.0), (-40, 0.0)):
        x = sign * 2.0 ** power
        y, mean, rstd = t.layer_norm(x, eps=eps)
        assert torch.equal(y, sign) and not mean.any() and (rstd == 2.0 ** -power).all()
        # dy along y has no gradient, dy = 1 none but in dbias
        for dy, want in ((sign, 0.0), (torch.ones_like(x), 0.0)):
            dx, _, db = t.layer_norm_backward(dy, x, mean, rstd, bias=True)
            assert (dx == want).all() and torch.equal(db, dy.sum(0))
    x = torch.full((3, cols), 2.0 ** (126 - math.ceil(math.log2(cols))), device="cuda")
    y, mean, _ = t.layer_norm(x)
    assert not y.any() and torch.equal(mean, x[:, 0])
