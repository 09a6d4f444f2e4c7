"""When OrthogonalMomentum takes a gradient and when it refuses, on the CPU with the operators in
plain torch: each gradient is applied once, and only one that backward has written."""
import pytest
import torch

import cpu_experts as C
from paper_2606_00539_amd import torch_experts as E

OFF = torch.tensor([0, 2, 5], dtype=torch.int32)


@pytest.fixture
def training(monkeypatch):
    C.patch(monkeypatch)
    units = E.ExpertUnits([("a", C.weight(2, 8, 16)), ("b", C.weight(2, 16, 8, seed=1))],
                          low_cost=False)
    opt = E.OrthogonalMomentum(units, lr=0.5, momentum=0.5)
    x = torch.randn(5, 16, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)

    def backward(only_a=False):
        y = units.linear("a", x, OFF)
        (y if only_a else units.linear("b", y, OFF)).float().sum().backward()
    return units, opt, backward


def state(units, opt):
    return [t.detach().clone() for t in (*units.weights, *opt.buffers.values())]


def refused(units, opt, match):
    before = state(units, opt)
    with pytest.raises(RuntimeError, match=match):
        opt.step()
    assert all(torch.equal(a, b) for a, b in zip(before, state(units, opt)))


def test_a_step_before_every_gradient_is_refused(training):
    units, opt, backward = training
    refused(units, opt, "a: no gradient")
    backward(only_a=True)
    refused(units, opt, "b: no gradient")
    backward()
    opt.step()


@pytest.mark.parametrize("controller_first", [True, False])
def test_a_gradient_is_applied_once(training, controller_first):
    units, opt, backward = training
    m = 0.0
    for _ in range(3):
        backward()
        backward()
        g = units.grads["a"].clone()
        if controller_first:
            units.step(1.1, 1.5)
        opt.step()
        if not controller_first:
            units.step(1.1, 1.5)
        m = 0.5 * m + g
        assert torch.equal(opt.buffers["a"], m)
        refused(units, opt, "no gradient")


def test_a_gradient_that_holds_an_applied_one_is_refused(training):
    units, opt, backward = training
    backward()
    opt.step()
    backward()                          # adds to what was applied
    refused(units, opt, "no gradient was started since")
    units.zero_grad()
    backward()
    g = units.grads["b"].clone()
    m = opt.buffers["b"].clone()
    opt.step()
    assert torch.equal(opt.buffers["b"], 0.5 * m + g)


def test_zero_grad_starts_the_gradients_anew(training):
    units, opt, backward = training
    backward()
    once = [g.clone() for g in units.grads.values()]
    units.zero_grad()
    with pytest.raises(RuntimeError, match="no gradient"):
        units.step(1.1, 1.5)
    backward()
    assert all(torch.equal(a, b) for a, b in zip(once, units.grads.values()))
