"""A mixture-of-experts layer's matrices as GNMR units, end to end on the expert
step's kernels: products grouped by expert, gated feed-forward blocks, the low-cost path
in INT8, weight gradients with the controller's sums of squares, clipping by its norms,
orthogonalised updates.

Argument marshalling and bookkeeping only: the products, the codes, the norms and
the updates run in libgnmr.
"""
from __future__ import annotations

import numpy as np
import torch

from . import torch_ops as ops
from .binding import GNMR_BUDGET_ACTIVE, Controller, gnmr_grouped_wgrad_num_partials
from .torch_units import clip_from_controller, clippable, torch_stream


def _readable(dy):
    """dy where the kernels can read it.  Autograd may bring any strides and alignment: a sum's
    gradient has a row stride of 0, a concatenation's starts anywhere (and may be contiguous)."""
    if (dy.stride(1) == 1 and dy.shape[1] <= dy.stride(0) < 1 << 22 and dy.stride(0) % 8 == 0 and
            dy.data_ptr() % 16 == 0):
        return dy
    return dy.clone(memory_format=torch.contiguous_format)


def _handle(stream):
    return int(getattr(stream, "cuda_stream", stream))


def _captured(stream):
    with torch.cuda.stream(stream):
        return torch.cuda.is_current_stream_capturing()


class _FirstDerivative(torch.autograd.Function):
    """dx where backward is itself recorded: it depends on `on`, and whoever asks how is refused
    (the kernels that made it are not recorded)."""

    @staticmethod
    def forward(ctx, dx, name, *on):
        ctx.name = name
        return dx.view_as(dx)

    @staticmethod
    def backward(ctx, g):
        raise RuntimeError(f"ExpertUnits.{ctx.name} has no second derivatives")


class _Use:
    """One use of matrix k in a product: what its weight gradient is formed from, between the
    backward of the product and that of the weight."""

    def __init__(self, units, k):
        self.units, self.k, self.rows = units, k, None

    def write(self):
        rows, self.rows = self.rows, None
        self.units._weight_grad(self.k, *rows)

    def product(self, x, weight, offsets):
        """W_e x[t], each expert on its path."""
        units, k = self.units, self.k
        if units.codes[k] is None:
            return ops.grouped_linear(x, weight, offsets)
        y = torch.empty(x.shape[0], weight.shape[1], dtype=x.dtype, device=x.device)
        mask = units.mask(k)
        ops.grouped_linear(x, weight, offsets, mask=mask, mask_value=1, out=y)
        ops.quantized_linear(x, *units.codes[k], offsets, mask=mask, mask_value=0, out=y)
        return y

    def gated(self, x, weight, offsets, activation, keep):
        """(h, pre) of a gated block, each expert on its path; pre None where it is not kept."""
        units, k = self.units, self.k
        if units.codes[k] is None:
            out = ops.gated_linear(x, weight, offsets, activation=activation, keep=keep)
            return out if keep else (out, None)
        both = weight.shape[1]
        h = torch.empty(x.shape[0], both // 2, dtype=x.dtype, device=x.device)
        pre = torch.empty(x.shape[0], both, dtype=x.dtype, device=x.device)
        mask = units.mask(k)
        ops.gated_linear(x, weight, offsets, mask=mask, mask_value=1, activation=activation, out=h,
                         pre=pre)
        ops.quantized_linear(x, *units.codes[k], offsets, mask=mask, mask_value=0, out=pre)
        ops.gated_activation(pre, offsets, mask=mask, mask_value=0, activation=activation, out=h)
        return h, pre


class _WeightUse(torch.autograd.Function):
    """An empty tensor between the weight and its product: autograd comes here only where a
    weight gradient is asked for, which the product itself cannot see."""

    @staticmethod
    def forward(ctx, weight, use):
        ctx.use = use
        return weight.new_empty(0)

    @staticmethod
    def backward(ctx, _):
        ctx.use.write()
        return None, None


class _ExpertLinear(torch.autograd.Function):
    """y[t] = W_e x[t]: in bf16 for the experts of A_t, in INT8 for the others.  Backward
    takes the products with the bf16 weights and the bf16 input on both paths (a
    straight-through gradient)."""

    @staticmethod
    def forward(ctx, x, weight, token, offsets, use):
        ctx.save_for_backward(x, weight, offsets)
        ctx.use = use
        return use.product(x, weight, offsets)

    @staticmethod
    def backward(ctx, dy):
        x, weight, offsets = ctx.saved_tensors
        rows, token = _readable(dy.detach()), None
        dx = ops.grouped_dgrad(rows, weight, offsets) if ctx.needs_input_grad[0] else None
        if ctx.needs_input_grad[2]:
            ctx.use.rows, token = (rows, x, offsets), rows.new_empty(0)
        if dx is not None and torch.is_grad_enabled():      # create_graph
            dx = _FirstDerivative.apply(dx, "linear", dy, weight)
        return dx, None, token, None, None


class _ExpertFeedForward(torch.autograd.Function):
    """y[t] = V_e (act(G_e x[t]) * (U_e x[t])), both matrices each on its expert's path.  Backward
    takes the products with the bf16 weights, and the derivatives at the products that
    forward had (a straight-through gradient)."""

    @staticmethod
    def forward(ctx, x, up, down, up_token, down_token, offsets, up_use, down_use, activation,
                keep):
        h, pre = up_use.gated(x, up, offsets, activation, keep)
        if keep:
            ctx.save_for_backward(x, up, down, offsets, h, pre)
        ctx.uses, ctx.activation = (up_use, down_use), activation
        return down_use.product(h, down, offsets)

    @staticmethod
    def backward(ctx, dy):
        x, up, down, offsets, h, pre = ctx.saved_tensors
        up_use, down_use = ctx.uses
        of_x, _, _, of_up, of_down = ctx.needs_input_grad[:5]
        rows, dx, tokens = _readable(dy.detach()), None, [None, None]
        if of_x or of_up:
            dpre = ops.gated_dgrad(rows, down, pre, offsets, activation=ctx.activation)
        if of_x:
            dx = ops.grouped_dgrad(dpre, up, offsets)
            if torch.is_grad_enabled():     # create_graph
                dx = _FirstDerivative.apply(dx, "feed_forward", dy, x, up, down)
        if of_up:
            up_use.rows, tokens[0] = (dpre, x, offsets), rows.new_empty(0)
        if of_down:
            down_use.rows, tokens[1] = (rows, h, offsets), rows.new_empty(0)
        return dx, None, None, *tokens, None, None, None, None, None


class ExpertUnits:
    """Expert weights ([experts, out, in] bf16 parameters) as units, one per expert and
    matrix, named "<name>.<expert>".

    `linear(name, x, offsets)` is the layer: rows of x sorted by expert, expert e's in
    [offsets[e], offsets[e + 1]) (int32, on the device; a router's output need not come
    to the host).  With low_cost, experts outside A_t run in INT8 (codes of the weights
    made by `refresh()`, which an optimiser calls after it has changed them); the
    controller's mask is read on the device when the kernels run.  `feed_forward(up, down, x,
    offsets)` is a gated block of two of the matrices, its gate and up projections one matrix
    ([experts, 2 hidden, in], the gate's rows first) and so one unit per expert.

    Backward writes the weight gradients itself, into `grads[name]` in grad_dtype, where it is
    asked for them (`torch.autograd.grad(loss, x)` leaves them alone),
    adding over the micro-batches since the last `step()` (or `zero_grad()`), and the sums of squares of
    what it stores; `step()` runs the controller from those.  weight.grad stays None.  Second
    derivatives are refused.
    """

    def __init__(self, named_weights, window: int = 5, max_o: int = 8, lock_len: int = 8,
                 eps: float = 1e-12, recoverable=None, budget_mode: int = GNMR_BUDGET_ACTIVE,
                 warmup_steps: int = 0, low_cost: bool = True, grad_dtype=torch.float32,
                 stream=None):
        self.names, self.weights, self.unit_names, first, parts = [], [], [], [0], [0]
        for name, w in named_weights:
            if w.dim() != 3 or w.dtype != torch.bfloat16 or not w.is_cuda or not w.is_contiguous():
                raise TypeError(f"{name}: the weight must be a contiguous bf16 [experts, out, in] "
                                "tensor on a HIP device")
            if self.weights and w.device != self.weights[0].device:
                raise ValueError(f"{name}: all weights must be on one device, {w.device} is not "
                                 f"{self.weights[0].device}")
            E, o, i = w.shape
            if o % 8 or i % 8:
                raise ValueError(f"{name}: features must be multiples of 8, got {o}x{i}")
            self.names.append(name)
            self.weights.append(w)
            self.unit_names += [f"{name}.{e}" for e in range(E)]
            first.append(first[-1] + E)
            parts.append(parts[-1] + E * gnmr_grouped_wgrad_num_partials(o, i))
        if not self.weights:
            raise ValueError("no expert weight given")
        if grad_dtype not in (torch.bfloat16, torch.float32):
            raise TypeError("grad_dtype must be torch.bfloat16 or torch.float32")
        self._index = {n: k for k, n in enumerate(self.names)}
        self._first, self._parts = first, parts
        device = self.device = self.weights[0].device
        self.partials = torch.zeros(parts[-1], dtype=torch.float32, device=device)
        self.grads = {n: torch.empty(w.shape, dtype=grad_dtype, device=device)
                      for n, w in zip(self.names, self.weights)}
        self._filled = [False] * len(self.weights)
        self._started = [0] * len(self.weights)     # gradients started, by matrix
        self._writers = [None] * len(self.weights)  # the stream that last wrote each, or its handle
        self._stepped = None                        # the stream of the last step: it reads the sums
        self._replayed = [False] * len(self.weights)    # written by a graph, unseen by the host
        U = first[-1]
        off = np.zeros(U + 1, np.int64)
        for k, w in enumerate(self.weights):
            n = (parts[k + 1] - parts[k]) // w.shape[0]
            off[first[k] + 1:first[k + 1] + 1] = parts[k] + n * np.arange(1, w.shape[0] + 1)
        rec = None
        if recoverable is not None:
            rec = np.array([1 if recoverable(u) else 0 for u in self.unit_names], np.uint8)
        with torch.cuda.device(device):         # a controller is the current device's
            self.ctl = Controller(U, window, max_o, lock_len, eps, np.zeros(U + 1, np.int64), [],
                                  [], None, rec, self._stream(stream), budget_mode, warmup_steps)
        self.ctl.bind_partials(off)
        self._mask = torch.as_tensor(_DeviceBytes(self.ctl, U), device=device)
        self.low_cost = bool(low_cost)
        self.codes = [None] * len(self.weights)
        self.refresh()

    def _stream(self, stream):
        """`stream`, or torch's current one on the weights' device when it is None."""
        return torch.cuda.current_stream(self.device) if stream is None else stream

    def mask(self, k):
        """The controller's mask over matrix k's experts (device memory of the controller)."""
        return self._mask[self._first[k]:self._first[k + 1]]

    def refresh(self) -> None:
        """The weights' INT8 codes again, after the weights have changed.  They stay where they
        are, for captured graphs and for what another stream is still reading."""
        if self.low_cost:
            self.codes = [ops.quantize_rows(w.detach(), out=c)
                          for w, c in zip(self.weights, self.codes)]

    def _use(self, name):
        """(weight, token, use) of a matrix in a product."""
        k = self._index[name]
        use, weight, token = _Use(self, k), self.weights[k], None
        if weight.requires_grad and torch.is_grad_enabled():
            token = _WeightUse.apply(weight, use)
        return weight, token, use

    def linear(self, name, x, offsets):
        weight, token, use = self._use(name)
        return _ExpertLinear.apply(x, weight, token, offsets, use)

    def feed_forward(self, up, down, x, offsets, activation="silu"):
        """The gated block y[t] = V_e (act(G_e x[t]) * (U_e x[t])) for the rows t of every expert e:
        matrix `up` is [G_e; U_e], [experts, 2 hidden, in], and `down` V_e, [experts, out, hidden];
        activation "silu" or "gelu".  As with torch's own operators, its backward pass is captured in a
        graph only while no autograd graph made outside the capture holds the same leaves."""
        a, b = self.weights[self._index[up]], self.weights[self._index[down]]
        if a.shape[0] != b.shape[0] or a.shape[1] != 2 * b.shape[2] or b.shape[2] % 8:
            raise ValueError(f"{up} and {down} must be [experts, 2 hidden, in] and [experts, out, "
                             f"hidden], hidden a multiple of 8, not {tuple(a.shape)} and "
                             f"{tuple(b.shape)}")
        keep = torch.is_grad_enabled() and any(t.requires_grad for t in (x, a, b))
        (a, a_token, a_use), (b, b_token, b_use) = self._use(up), self._use(down)
        return _ExpertFeedForward.apply(x, a, b, a_token, b_token, offsets, a_use, b_use, activation,
                                        keep)

    def _after_writers(self, stream, writers):
        """Work that follows on `stream` runs after the gradients' writers, or what reads them.
        (Backward runs where forward did, on several streams perhaps; autograd orders only what passes
        through it.)  A stream under capture waits only for others of its capture, which end with
        it."""
        for w in {_handle(w): w for w in writers if w is not None}.values():
            if _handle(w) != _handle(stream):
                stream, w = (torch_stream(t, self.device) for t in (stream, w))
                if _captured(stream) == _captured(w):
                    stream.wait_stream(w)

    def _weight_grad(self, k, dy, x, offsets):
        E, stream = self.weights[k].shape[0], self._stream(None)
        # (what follows a gradient's start is behind the step with that)
        self._after_writers(stream, [self._writers[k], None if self._filled[k] else self._stepped])
        ops.grouped_wgrad(dy, x, offsets, dw=self.grads[self.names[k]],
                          accumulate=self._filled[k],
                          partials=self.partials[self._parts[k]:self._parts[k + 1]].view(E, -1))
        self._writers[k] = stream
        self._replayed[k] |= torch.cuda.is_current_stream_capturing()
        self._started[k] += not self._filled[k]
        self._filled[k] = True

    def zero_grad(self) -> None:
        """The next backward starts the gradients anew, without a controller step."""
        self._filled = [False] * len(self.weights)

    def step(self, alpha_t: float, beta_t: float, stream=None) -> None:
        """One controller step from the gradients since the last one (asynchronous).  The next
        gradients wait for `stream`, which lives until then."""
        for n, done in zip(self.names, self._filled):
            if not done:
                raise RuntimeError(f"{n}: no gradient was written since the last step")
        stream = self._stream(stream)
        self._after_writers(stream, self._writers)
        self.ctl.step_from_partials(self.partials, alpha_t, beta_t, stream)
        self._stepped = stream
        self._filled = [False] * len(self.weights)

    def step_clipped(self, alpha_t: float, beta_t: float, max_norm: float, others=(),
                     eps: float = 1e-6, stream=None):
        """step(), and then the gradients, with `others` (more gradient tensors of the step), scaled in
        place to a global norm of at most max_norm.  The units' norms are those that the step has just
        made; only `others`, ready on `stream`, are read for the norm.  Returns it (a float64 scalar on the
        device, there on `stream`).  A unit's norm of 2^64 or more is infinite, and then everything is
        scaled by 0; values below 2^-75 do not count in it.  A call that is refused for `others` has not
        stepped.  What takes the gradients here next, an update or the next backward, waits for `stream`."""
        stream, gradients = self._stream(stream), list(self.grads.values())
        others = clippable(gradients, others, max_norm, eps, self.device)
        self.step(alpha_t, beta_t, stream)
        self._writers = [stream] * len(self.weights)
        return clip_from_controller(self.ctl, gradients, others, max_norm, eps, stream, self.device)

    def query(self, stream=None) -> dict:
        out = self.ctl.query(self._stream(stream))
        out["units"] = self.unit_names
        return out

    def recovery_set(self, stream=None) -> list:
        m = self.ctl.query(self._stream(stream))["mask"]
        return [u for u, a in zip(self.unit_names, m) if a]

    def close(self):
        self._mask = None
        self.codes = [None] * len(self.weights)
        self.ctl.close()


class _DeviceBytes:
    """The controller's mask as an array of device bytes; it keeps the controller."""

    def __init__(self, ctl, n):
        self.ctl = ctl
        self.__cuda_array_interface__ = {"shape": (n,), "typestr": "|u1", "version": 2,
                                         "data": (int(ctl.device_outputs()["mask"]), False)}


class OrthogonalMomentum:
    """Updates the weights of ExpertUnits with their orthogonalised momentum: per matrix
    m = momentum * m + g (fp32), W -= lr * max(1, out / in)^0.5 * orthogonalize(m), all
    experts of a matrix in one call; then the units' codes are made again.  Each gradient is
    taken once: `units.step()` or `units.zero_grad()` comes between an update and the next
    backward, else that would add to what was applied, and `step()` raises.  (A backward that was
    captured in a graph writes with every replay, which the host does not see: there nothing
    is asked.)"""

    def __init__(self, units, lr: float, momentum: float = 0.95, steps: int = 5,
                 coefficients=ops.COEFFICIENTS, eps: float = 1e-7):
        self.units, self.lr, self.momentum = units, float(lr), float(momentum)
        self.steps, self.coefficients, self.eps = steps, coefficients, eps
        self.buffers = {n: torch.zeros(g.shape, dtype=torch.float32, device=g.device)
                        for n, g in units.grads.items()}
        self._applied = [0] * len(units.weights)    # units._started of the last update

    @torch.no_grad()
    def step(self) -> None:
        for name, started, applied, replayed in zip(self.units.names, self.units._started,
                                                    self._applied, self.units._replayed):
            if started == applied and not replayed:
                raise RuntimeError(f"{name}: no gradient was started since the last update")
        self._applied = list(self.units._started)
        self.units._after_writers(self.units._stream(None), self.units._writers)
        for name, w in zip(self.units.names, self.units.weights):
            m = self.buffers[name]
            m.mul_(self.momentum).add_(self.units.grads[name])
            scale = max(1.0, w.shape[1] / w.shape[2]) ** 0.5
            w.sub_(ops.orthogonalize(m, self.steps, self.coefficients, self.eps, scale),
                   alpha=self.lr)
        self.units.refresh()
