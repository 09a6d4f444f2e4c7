"""What autograd may ask of ExpertUnits.feed_forward, on the CPU with the operators in plain torch."""
import pytest
import torch

import cpu_experts as C
from paper_2606_00539_amd import torch_experts as E

OFF = torch.tensor([0, 3, 3, 8], dtype=torch.int32)
H = 16


def act(kind):
    return {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[kind]


def gated_linear(x, w, offsets=None, activation="silu", keep=False):
    pre = C.grouped_linear(x, w, offsets)
    h = act(activation)(pre[:, :H]) * pre[:, H:]
    return (h, pre) if keep else h


def gated_dgrad(dy, w, pre, offsets=None, activation="silu"):
    d, p = C.grouped_dgrad(dy, w, offsets), pre.detach().requires_grad_()
    with torch.enable_grad():
        h = act(activation)(p[:, :H]) * p[:, H:]
    return torch.autograd.grad(h, p, d)[0]


@pytest.fixture
def block(monkeypatch):
    C.patch(monkeypatch)
    monkeypatch.setattr(E.ops, "gated_linear", gated_linear)
    monkeypatch.setattr(E.ops, "gated_dgrad", gated_dgrad)
    up, down = C.weight(3, 2 * H, 24), C.weight(3, 8, H, seed=1)
    g = torch.Generator().manual_seed(2)
    x = torch.randn(8, 24, generator=g).to(torch.bfloat16).requires_grad_()
    return E.ExpertUnits([("up", up), ("down", down)], low_cost=False), x, up, down


def reference(x, up, down, kind="silu"):
    out = []
    for e in range(3):
        p = x[OFF[e]:OFF[e + 1]].float() @ up[e].float().t()
        out.append((act(kind)(p[:, :H]) * p[:, H:]) @ down[e].float().t())
    return torch.cat(out)


@pytest.mark.parametrize("kind", ["silu", "gelu"])
def test_gradients_go_where_they_belong(block, kind):
    units, x, up, down = block
    y = units.feed_forward("up", "down", x, OFF, activation=kind)
    dy = torch.randn(8, 8, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    y.backward(dy)
    leaves = [t.detach().as_subclass(torch.Tensor).float().requires_grad_() for t in (x, up, down)]
    want = reference(*leaves, kind)
    want.backward(dy.float())
    for got, ref in ((y, want), (x.grad, leaves[0].grad), (units.grads["up"], leaves[1].grad),
                     (units.grads["down"], leaves[2].grad)):
        # five roundings of at most 2^-8 in a row
        assert (got.detach().float() - ref.detach()).norm() < 5 * 2.0 ** -8 * ref.norm()
    assert up.grad is None and down.grad is None
    first = {n: g.clone() for n, g in units.grads.items()}
    units.feed_forward("up", "down", x, OFF, activation=kind).backward(dy)
    for n, g in units.grads.items():
        torch.testing.assert_close(g, 2 * first[n])


def test_only_what_is_asked_for_is_written(block):
    units, x, up, down = block
    torch.autograd.grad(units.feed_forward("up", "down", x, OFF).float().sum(), x)
    assert units._filled == [False, False]
    with pytest.raises(RuntimeError, match="up: no gradient"):
        units.step(1.1, 1.5)
    down.requires_grad_(False)
    units.feed_forward("up", "down", x, OFF).float().sum().backward()
    assert units._filled == [True, False]
    units.zero_grad()
    down.requires_grad_()
    up.requires_grad_(False)
    x.requires_grad_(False)
    units.feed_forward("up", "down", x, OFF).float().sum().backward()
    assert units._filled == [False, True]


def test_what_is_kept(block, monkeypatch):
    """The products are kept only where backward can come."""
    units, x, up, down = block
    asked = []
    monkeypatch.setattr(E.ops, "gated_linear",
                        lambda *a, keep, **k: asked.append(keep) or gated_linear(*a, keep=keep, **k))
    units.feed_forward("up", "down", x, OFF)
    with torch.no_grad():
        units.feed_forward("up", "down", x, OFF)
    for t in (x, up, down):
        t.requires_grad_(False)
    units.feed_forward("up", "down", x, OFF)
    assert asked == [True, False, False]


@pytest.mark.parametrize("beside", [False, True])
def test_second_derivatives_are_refused(block, beside):
    units, x, up, down = block
    # of a sum, whose own gradient is a constant: the gradient depends on x all the same
    g, = torch.autograd.grad(units.feed_forward("up", "down", x, OFF).float().sum(), x,
                             create_graph=True)
    penalty = g.float().square().sum()
    if beside:
        penalty = penalty + x.float().square().sum()
    with pytest.raises(RuntimeError, match="feed_forward has no second derivatives"):
        penalty.backward()


def test_refusals(block):
    units, x, up, down = block
    for a, b in (("down", "up"), ("up", "up"), ("down", "down")):
        with pytest.raises(ValueError):
            units.feed_forward(a, b, x, OFF)
    with pytest.raises(KeyError):
        units.feed_forward("up", "other", x, OFF)
