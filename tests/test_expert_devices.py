"""ExpertUnits where the weights are not on the current device: the controller, its stream
and every buffer go with the weights.  On the CPU: devices are only noted."""
import contextlib

import numpy as np
import pytest
import torch

import cpu_experts as C
from paper_2606_00539_amd import torch_experts as E


class There(C.OnDevice):
    """A CPU tensor that says which HIP device it is on."""
    __torch_function__ = torch._C._disabled_torch_function_impl
    index = 1

    @property
    def device(self):
        return torch.device("cuda", self.index)


class Here(There):
    __torch_function__ = torch._C._disabled_torch_function_impl
    index = 0


def weight(kind, *shape):
    return torch.zeros(*shape, dtype=torch.bfloat16).as_subclass(kind)


class Noted:
    """torch, with the devices that it is asked for noted and nothing on them."""

    def __init__(self):
        self.asked, self.current = [], torch.device("cuda", 0)
        self.cuda = self

    def __getattr__(self, name):
        return getattr(torch, name)

    @contextlib.contextmanager
    def device(self, device):
        was, self.current = self.current, device
        yield
        self.current = was

    def current_stream(self, device=None):
        return ("stream of", self.current if device is None else device)

    def _on(self, f, *a, device, **kw):
        self.asked.append(device)
        return f(*a, **kw)

    def zeros(self, *a, **kw):
        return self._on(torch.zeros, *a, **kw)

    def empty(self, *a, **kw):
        return self._on(torch.empty, *a, **kw)

    def as_tensor(self, *a, **kw):
        return self._on(torch.as_tensor, *a, **kw)


@pytest.fixture
def noted(monkeypatch):
    C.patch(monkeypatch)
    t = Noted()

    class Controller(C.NotedController):
        def __init__(self, *args):
            super().__init__(*args)
            self.device = t.current

    monkeypatch.setattr(E, "torch", t)
    monkeypatch.setattr(E, "Controller", Controller)
    monkeypatch.setattr(torch.cuda, "current_stream", t.current_stream)
    return t


def test_the_controller_is_on_the_weights_device(noted):
    there = torch.device("cuda", 1)
    units = E.ExpertUnits([("a", weight(There, 2, 8, 16)), ("b", weight(There, 3, 16, 8))],
                          low_cost=False)
    assert units.ctl.device == there and set(noted.asked) == {there}
    assert any(c == ("stream of", there) for c in units.ctl.calls[0] if isinstance(c, tuple))
    units._filled = [True, True]
    units.step(1.1, 1.5)
    units.query()
    units.recovery_set()
    assert [c[-1] for c in units.ctl.calls[1:]] == [("stream of", there)] * 3
    units._filled = [True, True]
    units.step(1.1, 1.5, stream=17)
    assert units.ctl.calls[-1][-1] == 17
    assert noted.current == torch.device("cuda", 0)


def test_weights_of_several_devices_are_refused(noted):
    with pytest.raises(ValueError, match="b.*one device"):
        E.ExpertUnits([("a", weight(Here, 2, 8, 16)), ("b", weight(There, 2, 8, 16))],
                      low_cost=False)
