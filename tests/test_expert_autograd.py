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


def wgrad(dy, x):
    return torch.stack([dy[OFF[e]:OFF[e + 1]].float().t() @ x[OFF[e]:OFF[e + 1]].float()
                        for e in range(3)])


def test_an_input_gradient_alone_leaves_the_weights_gradient(layer):
    units, w, x = layer
    ones = torch.ones(8, 16)
    torch.autograd.grad(units.linear("m", x, OFF).float().sum(), x)
    with pytest.raises(RuntimeError, match="no gradient"):
        units.step(1.1, 1.5)
    # the next backward starts anew, from the same graph or another
    y = units.linear("m", x, OFF).float().sum()
    torch.autograd.grad(y, x, retain_graph=True)
    y.backward()
    want = wgrad(ones, x.detach())
    assert torch.equal(units.grads["m"], want)
    torch.autograd.grad(units.linear("m", x, OFF).float().sum(), x)
    y = units.linear("m", x, OFF).float().sum()
    y.backward(inputs=[x])
    assert torch.equal(units.grads["m"], want)
    units.linear("m", x, OFF).float().sum().backward()
    assert torch.equal(units.grads["m"], 2 * want)
    units.step(1.1, 1.5)
    assert torch.equal(units.ctl.calls[-1][1].view(3), (2 * want).square().sum((1, 2)))


def test_every_use_of_a_matrix_adds_its_gradient(layer):
    units, w, x = layer
    g = torch.Generator().manual_seed(2)
    dy = torch.randn(2, 8, 16, generator=g).to(torch.bfloat16)
    a, b = units.linear("m", x, OFF), units.linear("m", 2 * x, OFF)
    torch.autograd.backward([a, b], [dy[0], dy[1]])
    want = wgrad(dy[0], x.detach()) + wgrad(dy[1], 2 * x.detach())
    torch.testing.assert_close(units.grads["m"], want, rtol=1e-5, atol=1e-5)
    assert w.grad is None and x.grad is not None


def test_a_frozen_matrix_gets_no_gradient(layer):
    units, w, x = layer
    w.requires_grad_(False)
    units.linear("m", x, OFF).float().sum().backward()
    with pytest.raises(RuntimeError, match="no gradient"):
        units.step(1.1, 1.5)
    assert torch.equal(x.grad, torch.cat([torch.ones(OFF[e + 1] - OFF[e], 16).to(torch.bfloat16) @ w[e]
                                          for e in range(3)]))


def test_only_the_weights_gradient(layer):
    units, w, x = layer
    units.linear("m", x.detach(), OFF).float().sum().backward()
    assert torch.equal(units.grads["m"], wgrad(torch.ones(8, 16), x.detach()))


def test_checkpointed_layers_write_their_gradient_once(layer):
    from torch.utils.checkpoint import checkpoint

    units, w, x = layer
    want = wgrad(torch.ones(8, 16), x.detach())
    for reentrant in (False, True):
        units.zero_grad()
        y = checkpoint(lambda v: units.linear("m", v, OFF), x, use_reentrant=reentrant)
        y.float().sum().backward()
        assert torch.equal(units.grads["m"], want)


def test_without_autograd_nothing_is_kept(layer):
    units, w, x = layer
    with torch.no_grad():
        y = units.linear("m", x, OFF)
    assert not y.requires_grad
    assert torch.equal(y, reference(x.detach(), w.detach().as_subclass(torch.Tensor)))
