"""Where steps and step_clipped run, and what waits for them, on the CPU with streams that only
note what waits for what."""
import contextlib

import pytest
import torch

import cpu_experts as C
from paper_2606_00539_amd import torch_experts as E
from paper_2606_00539_amd import torch_ops, torch_units

OFF = torch.tensor([0, 2, 5], dtype=torch.int32)


class Stream:
    def __init__(self, handle, log):
        self.cuda_stream, self.log = handle, log

    def wait_stream(self, other):
        self.log.append((self.cuda_stream, "waits for", other.cuda_stream))


class Machine:
    """Streams, units of two matrices and their update, and the order of what they do."""

    def __init__(self, monkeypatch):
        C.patch(monkeypatch)
        self.log, self.now = [], [1]
        monkeypatch.setattr(torch.cuda, "current_stream",
                            lambda device=None: Stream(self.now[-1], self.log))
        # (torch makes a stream of its own of handle 0)
        monkeypatch.setattr(torch.cuda, "ExternalStream",
                            lambda handle, device=None: Stream(handle or 1000, self.log))
        monkeypatch.setattr(torch.cuda, "default_stream",
                            lambda device=None: Stream(0, self.log))
        monkeypatch.setattr(torch.cuda, "stream", self.on)
        monkeypatch.setattr(torch_units, "_DeviceNorms", lambda ctl: [0.0])
        monkeypatch.setattr(torch_ops, "clip_gradients", self.noted("clips"))
        monkeypatch.setattr(E.ops, "orthogonalize", lambda m, *a: (self.note("updates"), m)[1])
        wgrad = E.ops.grouped_wgrad
        monkeypatch.setattr(E.ops, "grouped_wgrad",
                            lambda *a, **kw: (self.note("writes"), wgrad(*a, **kw))[1])
        self.units = E.ExpertUnits([("m", C.weight(2, 8, 16)), ("n", C.weight(2, 16, 16))],
                                   low_cost=False)
        self.units.device = torch.device("cpu")
        self.units.ctl.step_from_partials = lambda *a: self.log.append(
            (int(getattr(a[3], "cuda_stream", a[3])), "steps"))
        self.opt = E.OrthogonalMomentum(self.units, lr=0.1)
        self.x = torch.ones(5, 16, dtype=torch.bfloat16)

    @contextlib.contextmanager
    def on(self, stream):
        self.now.append(stream.cuda_stream)
        yield
        self.now.pop()

    def note(self, what):
        self.log.append((self.now[-1], what))

    def noted(self, what):
        return lambda *a, **kw: self.note(what)

    def backward(self, stream):
        with self.on(Stream(stream, self.log)):
            for name in self.units.names:
                self.units.linear(name, self.x, OFF).float().sum().backward()

    def streams(self, given):
        """`given` as the caller may hand it over: an object or a handle."""
        return [Stream(given, self.log), given]


@pytest.fixture
def machine(monkeypatch):
    return Machine(monkeypatch)


@pytest.mark.parametrize("how", [0, 1])
def test_the_update_waits_for_the_clipping(machine, how):
    machine.backward(1)
    machine.units.step_clipped(1.1, 1.5, 1.0, stream=machine.streams(7)[how])
    machine.opt.step()
    assert machine.log == [(1, "writes"), (1, "writes"), (7, "waits for", 1), (7, "steps"),
                           (7, "clips"), (1, "waits for", 7), (1, "updates"), (1, "updates")]


@pytest.mark.parametrize("how", [0, 1])
def test_the_next_gradients_wait_for_the_clipping(machine, how):
    machine.backward(1)
    machine.units.step_clipped(1.1, 1.5, 1.0, stream=machine.streams(7)[how])
    del machine.log[:]
    machine.backward(5)
    assert machine.log == [(5, "waits for", 7), (5, "writes")] * 2
    machine.units.step_clipped(1.1, 1.5, 1.0, stream=machine.streams(7)[how])
    assert machine.log[4:] == [(7, "waits for", 5), (7, "steps"), (7, "clips")]


@pytest.mark.parametrize("how", [0, 1])
def test_the_next_sums_of_squares_wait_for_the_step(machine, how):
    """The controller reads those of the last gradients, where the next ones go."""
    machine.backward(1)
    machine.units.step(1.1, 1.5, stream=machine.streams(7)[how])
    del machine.log[:]
    machine.backward(1)
    assert machine.log == [(1, "waits for", 7), (1, "writes")] * 2
    del machine.log[:]
    machine.backward(1)                 # another micro-batch, behind the first
    assert machine.log == [(1, "writes")] * 2
    machine.units.step(1.1, 1.5)
    del machine.log[:]
    machine.backward(1)
    assert machine.log == [(1, "writes")] * 2


def test_one_stream_waits_for_nothing(machine):
    for _ in range(2):
        machine.backward(1)
        machine.units.step_clipped(1.1, 1.5, 1.0)
        machine.opt.step()
    assert not any("waits for" in e for e in machine.log)


def test_handle_0_is_the_default_stream(machine):
    """step and step_clipped of the default stream's handle run there, and wait there."""
    machine.backward(1)
    machine.units.step_clipped(1.1, 1.5, 1.0, stream=0)
    assert machine.log[2:] == [(0, "waits for", 1), (0, "steps"), (0, "clips")]
    machine.backward(5)
    del machine.log[:]
    machine.units.step(1.1, 1.5, stream=0)
    assert machine.log == [(0, "waits for", 5), (0, "steps")]


@pytest.mark.parametrize("kind", ["TorchUnits", "FusedWgradUnits"])
def test_other_units_clip_where_they_step(machine, kind):
    units = object.__new__(getattr(torch_units, kind))
    m = torch.nn.Linear(4, 3)
    m.weight.grad = torch.ones(3, 4)
    units.modules, units.params, units.param_names = [m], [m.weight], ["w"]
    units.unit_names, units._produced, units.partials = ["w"], [m.weight.grad.data_ptr()], None
    on = []

    class Steps:
        def step(self, alpha, beta, seg_ptr, stream):
            on.append(int(getattr(stream, "cuda_stream", stream)))

        def step_from_partials(self, partials, alpha, beta, stream):
            on.append(int(getattr(stream, "cuda_stream", stream)))
    units.ctl = Steps()
    for k, given in enumerate((None, 0, 7, Stream(9, machine.log))):
        units._produced = [m.weight.grad.data_ptr()]
        units.step_clipped(1.1, 1.5, 1.0, stream=given)
        assert machine.log[-1] == (on[k], "clips")
    assert on == [1, 0, 7, 9]
