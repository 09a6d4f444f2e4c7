"""ExpertUnits on the CPU: its bookkeeping and autograd with the operators in plain torch and
a controller that only notes its calls."""
import contextlib

import numpy as np
import torch

from paper_2606_00539_amd import torch_experts as E


class OnDevice(torch.Tensor):
    """A CPU tensor that says that it is on a HIP device."""
    __torch_function__ = torch._C._disabled_torch_function_impl
    is_cuda = True


def weight(*shape, seed=0):
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(*shape, generator=g) / shape[-1] ** 0.5).to(torch.bfloat16)
    return w.as_subclass(OnDevice).requires_grad_()


class TheStream:
    """The one stream there is."""
    cuda_stream = 0


class NotedController:
    def __init__(self, *args):
        self.calls = [("init",) + args]

    def bind_partials(self, off):
        pass

    def step_from_partials(self, partials, alpha, beta, stream):
        self.calls.append(("step", partials.clone(), stream))

    def query(self, stream=None):
        self.calls.append(("query", stream))
        return {"mask": [0]}

    def close(self):
        self.calls.append(("close",))


def _rows(rows, w, offsets, product):
    out = torch.zeros(len(rows), product(rows[:0], w[0]).shape[1], dtype=rows.dtype)
    for e in range(len(w)):
        a, b = int(offsets[e]), int(offsets[e + 1])
        out[a:b] = product(rows[a:b], w[e])
    return out


def grouped_linear(x, w, offsets=None, **kw):
    return _rows(x.detach(), w.detach(), offsets, lambda r, m: r @ m.t())


def grouped_dgrad(dy, w, offsets=None, **kw):
    return _rows(dy.detach(), w.detach(), offsets, lambda r, m: r @ m)


def grouped_wgrad(dy, x, offsets, dw, accumulate=False, partials=None):
    if not accumulate:
        dw.zero_()
    for e in range(len(dw)):
        a, b = int(offsets[e]), int(offsets[e + 1])
        dw[e] += dy[a:b].detach().to(dw.dtype).t() @ x[a:b].detach().to(dw.dtype)
        partials[e] = dw[e].float().square().sum()
    return dw, partials


def orthogonalize(x, steps=5, coefficients=None, eps=1e-7, scale=1.0):
    return (scale * torch.sign(x)).to(torch.bfloat16)


def patch(monkeypatch):
    """Puts the plain forms in place of what needs a device."""
    monkeypatch.setattr(E, "Controller", NotedController)
    monkeypatch.setattr(E, "_DeviceBytes", lambda ctl, n: np.zeros(n, np.uint8))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: TheStream)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "stream", lambda stream: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "device", lambda device: contextlib.nullcontext())
    for f in (grouped_linear, grouped_dgrad, grouped_wgrad, orthogonalize):
        monkeypatch.setattr(E.ops, f.__name__, f)
