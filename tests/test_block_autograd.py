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


def test_one_matrix_as_both(monkeypatch):
    """[experts, 2 hidden, hidden] is up and down at once: its gradient is the sum of both."""
    C.patch(monkeypatch)
    monkeypatch.setattr(E.ops, "gated_linear", gated_linear)
    monkeypatch.setattr(E.ops, "gated_dgrad", gated_dgrad)
    w = C.weight(3, 2 * H, H)
    units = E.ExpertUnits([("m", w)], low_cost=False)
    g = torch.Generator().manual_seed(4)
    x = torch.randn(8, H, generator=g).to(torch.bfloat16).requires_grad_()
    dy = torch.randn(8, 2 * H, generator=g).to(torch.bfloat16)
    units.feed_forward("m", "m", x, OFF).backward(dy)
    leaves = [t.detach().as_subclass(torch.Tensor).float().requires_grad_() for t in (x, w)]
    reference(leaves[0], leaves[1], leaves[1]).backward(dy.float())
    for got, ref in ((x.grad, leaves[0].grad), (units.grads["m"], leaves[1].grad)):
        assert (got.float() - ref).norm() < 5 * 2.0 ** -8 * ref.norm()


class Steps:
    def __init__(self):
        self.steps = 0

    def step(self, *a, **kw):
        self.steps += 1

    step_from_partials = step


def bad_others(grad):
    f = torch.zeros(12)
    return [([None], TypeError), ([f.half()], TypeError), ([f.view(3, 4).t()], TypeError),
            ([f.to("meta")], TypeError), ([f, f], RuntimeError), ([f[:8], f[4:]], RuntimeError),
            ([grad], RuntimeError), ([grad.view(-1)[3:5]], RuntimeError)]


def check_step_clipped(units, grad, step):
    """What clipping refuses is refused before the controller has stepped."""
    for others, error in bad_others(grad):
        with pytest.raises(error):
            units.step_clipped(1.1, 1.5, 1.0, others=others)
    for kw in ({"max_norm": -1.0}, {"max_norm": float("nan")}, {"max_norm": 1.0, "eps": -1.0},
               {"max_norm": 1.0, "eps": float("inf")}):
        with pytest.raises(ValueError):
            units.step_clipped(1.1, 1.5, **kw)
    assert step.steps == 0


def test_a_refused_step_clipped_has_not_stepped(block, monkeypatch):
    units, x, up, down = block
    units.feed_forward("up", "down", x, OFF).float().sum().backward()
    units.device, units.ctl = torch.device("cpu"), Steps()
    check_step_clipped(units, units.grads["up"], units.ctl)
    assert units._filled == [True, True]
    clipped = []
    monkeypatch.setattr(E, "clip_from_controller", lambda *a: clipped.append(a))
    other = torch.ones(3)
    units.step_clipped(1.1, 1.5, 1.0, others=(t for t in [other]))
    assert units.ctl.steps == 1 and clipped[0][1:3] == (list(units.grads.values()), [other])


@pytest.mark.parametrize("kind", ["TorchUnits", "FusedWgradUnits"])
def test_a_refused_step_clipped_of_other_units_has_not_stepped(kind, monkeypatch):
    from paper_2606_00539_amd import torch_units as U

    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: C.TheStream)
    units = object.__new__(getattr(U, kind))
    m = torch.nn.Linear(4, 3)
    m.weight.grad = torch.ones(3, 4)
    units.modules, units.params, units.param_names, units.ctl = [m], [m.weight], ["w"], Steps()
    units._produced, units.partials = [m.weight.grad.data_ptr()], None
    check_step_clipped(units, m.weight.grad, units.ctl)
    monkeypatch.setattr(U, "clip_from_controller", lambda *a: None)
    units.step_clipped(1.1, 1.5, 1.0, others=[torch.ones(3)])
    assert units.ctl.steps == 1
