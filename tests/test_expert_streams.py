"""The order between streams that ExpertUnits keeps for its gradients, on the CPU with streams
that only note what waits for what."""
import pytest
import torch

import cpu_experts as C
from paper_2606_00539_amd import torch_experts as E

OFF = torch.tensor([0, 2, 5], dtype=torch.int32)


class Stream:
    def __init__(self, handle, log):
        self.cuda_stream, self.log = handle, log

    def wait_stream(self, other):
        self.log.append((self.cuda_stream, "waits for", other.cuda_stream))


@pytest.fixture
def streams(monkeypatch):
    C.patch(monkeypatch)
    log, now = [], [1]
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(now[0], log))
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: Stream(handle, log))
    wgrad = E.ops.grouped_wgrad

    def noted(*a, **kw):
        log.append((now[0], "adds" if kw["accumulate"] else "writes"))
        return wgrad(*a, **kw)
    monkeypatch.setattr(E.ops, "grouped_wgrad", noted)
    units = E.ExpertUnits([("m", C.weight(2, 8, 16))], low_cost=False)
    step = units.ctl.step_from_partials
    units.ctl.step_from_partials = lambda *a: (log.append((a[3], "steps")), step(*a))
    x = torch.ones(5, 16, dtype=torch.bfloat16)

    def backward(stream):
        now[0] = stream
        units.linear("m", x, OFF).float().sum().backward()
        now[0] = 1
    return units, backward, log


def test_one_stream_waits_for_nothing(streams):
    units, backward, log = streams
    for _ in range(2):
        backward(1)
        backward(1)
        units.step(1.1, 1.5)
        E.OrthogonalMomentum(units, lr=0.1).step()
    assert not any("waits for" in e for e in log)


def test_gradients_of_two_streams_are_added_in_order(streams):
    units, backward, log = streams
    backward(5)
    backward(6)
    backward(6)
    assert log == [(5, "writes"), (6, "waits for", 5), (6, "adds"), (6, "adds")]


# another stream by torch's current one, as an object and as a handle
@pytest.mark.parametrize("how", ["current", "stream", "handle"])
def test_a_step_waits_for_the_gradients(streams, how):
    units, backward, log = streams
    backward(5)
    given = {"current": None, "stream": Stream(7, log), "handle": 7}[how]
    units.step(1.1, 1.5, stream=given)
    on = 1 if how == "current" else 7
    assert log[1] == (on, "waits for", 5) and log[2][1] == "steps" and len(log) == 3


def test_an_update_waits_for_the_gradients(streams, monkeypatch):
    units, backward, log = streams
    opt = E.OrthogonalMomentum(units, lr=0.1)
    backward(5)
    monkeypatch.setattr(E.ops, "orthogonalize", lambda m, *a: (log.append("updates"), m)[1])
    opt.step()
    assert log == [(5, "writes"), (1, "waits for", 5), "updates"]


@pytest.fixture
def capture(monkeypatch, streams):
    """Streams that are being captured."""
    on = set()
    current = torch.cuda.current_stream

    class Under:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.stream)

        def __exit__(self, *exc):
            monkeypatch.setattr(torch.cuda, "current_stream", current)
    monkeypatch.setattr(torch.cuda, "stream", Under)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing",
                        lambda: torch.cuda.current_stream().cuda_stream in on)
    return on


def test_a_capture_does_not_wait_for_what_is_outside_it(streams, capture):
    """Such a wait would end the capture; what came before it is its caller's to order."""
    units, backward, log = streams
    backward(5)                                         # a warm-up
    units.step(1.1, 1.5, stream=Stream(5, log))
    capture |= {6, 7}
    backward(6)
    backward(7)                                         # two streams of one capture
    units.step(1.1, 1.5, stream=Stream(6, log))
    capture.clear()
    backward(6)
    units.step(1.1, 1.5, stream=Stream(8, log))
    waits = [e for e in log if "waits for" in e]
    assert waits == [(7, "waits for", 6), (6, "waits for", 7), (6, "waits for", 7),
                     (8, "waits for", 6)]


def test_a_captured_gradient_is_new_with_every_replay(streams, capture):
    """The host does not see replays, so the optimiser does not ask for a backward between them."""
    units, backward, log = streams
    opt = E.OrthogonalMomentum(units, lr=0.1)
    capture.add(6)
    backward(6)
    capture.clear()
    for _ in range(3):
        opt.step()                                      # behind a replay each
    backward(1)
    opt.step()
