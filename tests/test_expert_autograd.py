"""What autograd may ask of ExpertUnits.linear, on the CPU with the operators in plain torch."""
import pytest
import torch

import cpu_experts as C
from paper_2606_00539_amd import torch_experts as E

OFF = torch.tensor([0, 3, 3, 8], dtype=torch.int32)


@pytest.fixture
def layer(monkeypatch):
    C.patch(monkeypatch)
    w = C.weight(3, 16, 24)
    g = torch.Generator().manual_seed(1)
    x = torch.randn(8, 24, generator=g).to(torch.bfloat16).requires_grad_()
    return E.ExpertUnits([("m", w)], low_cost=False), w, x


def reference(x, w):
    return torch.cat([x[OFF[e]:OFF[e + 1]] @ w[e].t() for e in range(3)])


# of a sum, whose own gradient is a constant, and of a sum of squares
@pytest.mark.parametrize("loss", [lambda y: y.float().sum(), lambda y: y.float().square().sum()])
@pytest.mark.parametrize("beside", [False, True])
def test_second_derivatives_are_refused(layer, loss, beside):
    units, w, x = layer
    total = loss(units.linear("m", x, OFF))
    g, = torch.autograd.grad(total, x, create_graph=True)
    plain = torch.nn.Parameter(w.detach().as_subclass(torch.Tensor).clone())
    want, = torch.autograd.grad(loss(reference(x, plain)), x)
    assert torch.equal(g, want)
    penalty = g.float().square().sum()
    if beside:
        penalty = penalty + x.float().square().sum()
    with pytest.raises(RuntimeError, match="second derivatives"):
        penalty.backward()


def test_a_gradient_that_nothing_depends_on_has_no_history(layer):
    units, w, x = layer
    w.requires_grad_(False)
    g, = torch.autograd.grad(units.linear("m", x, OFF).float().sum(), x, create_graph=True)
    assert not g.requires_grad
