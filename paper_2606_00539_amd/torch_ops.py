"""The expert step's and a gated block's operators on PyTorch tensors.

  grouped_linear, grouped_dgrad, grouped_wgrad   products grouped by expert
  quantize_rows, quantized_linear                the INT8 low-cost path
  orthogonalize                                  the Newton-Schulz update
  gated_linear, gated_activation, gated_dgrad    gated feed-forward by expert
  layer_norm, layer_norm_backward                layer norm of rows
  clip_gradients                                 the global norm, and clipping by it

Rows (tokens) lie sorted by expert: expert e has rows [offsets[e], offsets[e + 1])
of int32 device `offsets`; rows from offsets[-1] on belong to nobody and give 0.
With `mask` (device bytes or bools, one per expert) only experts whose entry is
`mask_value` are computed, and the outputs of the others stay as they were, so
such a call takes the tensor to write to.

Argument marshalling only: everything runs in libgnmr, on torch's current stream
of the tensors' device.  Nothing here is recorded by autograd (ExpertUnits.linear and
.feed_forward in torch_experts.py and LayerNorm in torch_layers.py are).
"""
from __future__ import annotations

import functools

import torch

from . import binding as B

_T = torch.Tensor
_DTYPES = {torch.bfloat16: B.GNMR_BF16, torch.float32: B.GNMR_F32}
_num_partials = functools.lru_cache(None)(B.gnmr_grouped_wgrad_num_partials)
_clip_workspace = functools.lru_cache(None)(B.gnmr_clip_gradients_workspace)
_norm_workspace = functools.lru_cache(1024)(B.gnmr_layer_norm_backward_workspace)
_ACTIVATIONS = {"silu": B.GNMR_ACT_SILU, "gelu": B.GNMR_ACT_GELU}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _matrix(name, t, dtype, cols=None):
    """A 2-d tensor whose rows the kernels can read where they lie."""
    if t.dim() != 2 or t.dtype != dtype or not t.is_cuda:
        raise TypeError(f"{name} must be a 2-d {dtype} tensor on a HIP device")
    if cols is not None and t.shape[1] != cols:
        raise ValueError(f"{name} must have {cols} columns, not {t.shape[1]}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}'s rows must be contiguous")
    return t


def _stride(t):
    """Elements between rows; a single row's stride means nothing to torch."""
    return t.stride(0) if t.shape[0] > 1 else -(-t.shape[1] // 8) * 8


def _weights(name, t, dtype):
    if t.dim() != 3 or t.dtype != dtype or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous [experts, out, in] {dtype} tensor on a HIP "
                        "device")
    return t


def _of(experts, offsets, mask, like):
    if offsets is None and experts != 1:
        raise ValueError("offsets may be left out only with one expert")
    if offsets is not None and (offsets.dtype != torch.int32 or offsets.device != like.device or
                                offsets.shape != (experts + 1,) or not offsets.is_contiguous()):
        raise TypeError("offsets must be a contiguous int32 tensor of experts + 1 entries on the "
                        "rows' device")
    if mask is not None and (mask.dtype not in (torch.uint8, torch.bool) or
                             mask.device != like.device or mask.shape != (experts,) or
                             not mask.is_contiguous()):
        raise TypeError("mask must be a contiguous uint8 or bool tensor of an entry per expert on "
                        "the rows' device")


def _same_device(like, *tensors):
    for t in tensors:
        if t is not None and t.device != like.device:
            raise ValueError("all tensors must be on one device")


def _output(out, mask, rows, cols, like):
    if out is None:
        if mask is not None:
            raise ValueError("with a mask, out is needed: the other experts' rows stay in it")
        return torch.empty(rows, cols, dtype=torch.bfloat16, device=like.device)
    _matrix("out", out, torch.bfloat16, cols)
    if out.shape[0] != rows:
        raise ValueError(f"out must have {rows} rows, not {out.shape[0]}")
    return out


class _Here:
    """The context of a call on the current device (torch.cuda.device takes longer than
    a small call's marshalling)."""

    def __enter__(self):
        pass

    def __exit__(self, *exc):
        pass


_HERE = _Here()
# the handle alone, without the object around it that takes ten times as long to make
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _on(t):
    """(context, stream): t's device made current, and torch's current stream on it."""
    index = t.device.index
    if index == torch.cuda.current_device():
        return _HERE, _raw_stream(index)
    return torch.cuda.device(index), _raw_stream(index)


def grouped_linear(x, w, offsets=None, mask=None, mask_value=1, out=None):
    """y[t] = W_e x[t] for the rows t of every expert e.  x: bf16 [rows, in], w: bf16
    [experts, out, in]; returns bf16 [rows, out]."""
    E, o, i = _weights("w", w, torch.bfloat16).shape
    _matrix("x", x, torch.bfloat16, i)
    _of(E, offsets, mask, x)
    y = _output(out, mask, x.shape[0], o, x)
    _same_device(x, w, y)
    device, stream = _on(x)
    with device:
        B.gnmr_grouped_linear(x, _stride(x), w, y, _stride(y), x.shape[0], E, o, i, offsets, mask,
                              mask_value, stream)
    return y


def grouped_dgrad(dy, w, offsets=None, mask=None, mask_value=1, out=None):
    """dx[t] = W_e^T dy[t], the gradient of grouped_linear's x."""
    E, o, i = _weights("w", w, torch.bfloat16).shape
    _matrix("dy", dy, torch.bfloat16, o)
    _of(E, offsets, mask, dy)
    dx = _output(out, mask, dy.shape[0], i, dy)
    _same_device(dy, w, dx)
    device, stream = _on(dy)
    with device:
        B.gnmr_grouped_dgrad(dy, _stride(dy), w, dx, _stride(dx), dy.shape[0], E, o, i, offsets,
                             mask, mask_value, stream)
    return dx


def grouped_wgrad(dy, x, offsets=None, mask=None, mask_value=1, dw=None, accumulate=False,
                  dtype=torch.bfloat16, partials=None):
    """(dw, partials): dw[e] = sum over e's rows of dy[t] x[t]^T, in `dtype` (bf16 or
    fp32), and the sums of its squares over 128 x 128 blocks, [experts, blocks] fp32
    (Controller.bind_partials / step_from_partials take them flat).  With accumulate
    the product is added to the `dw` given."""
    E = 1 if offsets is None else offsets.numel() - 1
    _matrix("dy", dy, torch.bfloat16)
    _matrix("x", x, torch.bfloat16)
    if x.shape[0] != dy.shape[0]:
        raise ValueError("dy and x must have the same rows")
    o, i = dy.shape[1], x.shape[1]
    _of(E, offsets, mask, dy)
    if dw is None:
        if accumulate or mask is not None:
            raise ValueError("accumulate and mask need the dw they leave values in")
        if dtype not in _DTYPES:
            raise TypeError("dtype must be torch.bfloat16 or torch.float32")
        dw = torch.empty(E, o, i, dtype=dtype, device=dy.device)
    elif dw.shape != (E, o, i) or dw.dtype not in _DTYPES or not dw.is_contiguous():
        raise TypeError(f"dw must be a contiguous bf16 or fp32 tensor of shape {(E, o, i)}")
    n = _num_partials(o, i)
    if partials is None:
        if mask is not None:
            raise ValueError("with a mask, partials is needed: the other experts' stay in it")
        partials = torch.empty(E, n, dtype=torch.float32, device=dy.device)
    elif partials.numel() != E * n or partials.dtype != torch.float32 or \
            not partials.is_contiguous():
        raise TypeError(f"partials must be a contiguous fp32 tensor of {E * n} entries")
    _same_device(dy, x, dw, partials)
    device, stream = _on(dy)
    with device:
        B.gnmr_grouped_wgrad(dy, _stride(dy), x, _stride(x), dw, _DTYPES[dw.dtype], accumulate,
                             partials, dy.shape[0], E, o, i, offsets, mask, mask_value, stream)
    return dw, partials


def quantize_rows(x, out=None):
    """(codes, scale): symmetric INT8 codes of x's rows (over its last dimension; any
    leading ones) and the fp32 scale of each; `out` is such a pair to write them to."""
    if x.dtype not in _DTYPES or not x.is_cuda or x.dim() < 2:
        raise TypeError("x must be a bf16 or fp32 tensor of rows on a HIP device")
    flat = x if x.dim() == 2 else x.reshape(-1, x.shape[-1])
    _matrix("x", flat, x.dtype)
    if out is None:
        codes = torch.empty(x.shape, dtype=torch.int8, device=x.device)
        scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    else:
        codes, scale = out
        for name, t, shape, dtype in (("codes", codes, x.shape, torch.int8),
                                      ("scale", scale, x.shape[:-1], torch.float32)):
            if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
                raise TypeError(f"{name} must be a contiguous {dtype} tensor of shape "
                                f"{tuple(shape)}")
        _same_device(x, codes, scale)
    device, stream = _on(x)
    with device:
        B.gnmr_quantize_rows(flat, _DTYPES[x.dtype], _stride(flat), codes, scale, flat.shape[0],
                             flat.shape[1], stream)
    return codes, scale


def quantized_linear(x, codes, scale, offsets=None, mask=None, mask_value=0, out=None,
                     x_scale=None):
    """y = x W^T in 8-bit integers: W as codes ([out, in], or [experts, out, in] with
    offsets) and scale ([out], [experts, out]) from quantize_rows.  x: bf16 rows,
    quantised per token on the way, or int8 codes with their x_scale.  Returns bf16
    [rows, out]."""
    c = codes if codes.dim() == 3 else codes[None]
    E, o, i = _weights("codes", c, torch.int8).shape
    if scale.shape != codes.shape[:-1] or scale.dtype != torch.float32 or \
            not scale.is_contiguous():
        raise TypeError("scale must be a contiguous fp32 tensor of an entry per channel")
    _matrix("x", x, torch.bfloat16 if x_scale is None else torch.int8, i)
    if x_scale is not None and (x_scale.shape != x.shape[:1] or x_scale.dtype != torch.float32 or
                                not x_scale.is_contiguous()):
        raise TypeError("x_scale must be a contiguous fp32 tensor of an entry per row")
    _of(E, offsets, mask, x)
    rows = x.shape[0]
    y = _output(out, mask, rows, o, x)
    _same_device(x, codes, scale, y, x_scale)
    n = 0 if x_scale is not None else B.gnmr_quantized_linear_workspace(rows, i)
    work = torch.empty(n, dtype=torch.uint8, device=x.device) if n else None
    device, stream = _on(x)
    with device:
        B.gnmr_quantized_linear(x, _stride(x), x_scale, c, scale, y, _stride(y), rows, E, o, i,
                                work, n, offsets, mask, mask_value, stream)
    return y


def orthogonalize(x, steps=5, coefficients=COEFFICIENTS, eps=1e-7, scale=1.0, out=None):
    """The updates x (bf16 or fp32, [rows, cols] or [count, rows, cols]) with their
    singular values driven to about 1 by Newton-Schulz steps, times scale, in bf16."""
    if x.dim() not in (2, 3) or x.dtype not in _DTYPES or not x.is_cuda or not x.is_contiguous():
        raise TypeError("x must be a contiguous bf16 or fp32 tensor of one matrix or a batch on a "
                        "HIP device")
    if out is None:
        out = torch.empty(x.shape, dtype=torch.bfloat16, device=x.device)
    elif out.shape != x.shape or out.dtype != torch.bfloat16 or not out.is_contiguous() or \
            out.device != x.device:
        raise TypeError("out must be a contiguous bf16 tensor of x's shape and device")
    count, (m, n) = (1 if x.dim() == 2 else x.shape[0]), x.shape[-2:]
    size = B.gnmr_orthogonalize_workspace(m, n, count)
    work = torch.empty(size, dtype=torch.uint8, device=x.device) if size else None
    device, stream = _on(x)
    with device:
        B.gnmr_orthogonalize(x, _DTYPES[x.dtype], out, m, n, count, steps, coefficients, eps,
                             scale, work, size, stream)
    return out


def _activation(name):
    if name not in _ACTIVATIONS:
        raise ValueError(f"activation must be one of {', '.join(_ACTIVATIONS)}, not {name!r}")
    return _ACTIVATIONS[name]


def gated_linear(x, w, offsets=None, mask=None, mask_value=1, activation="silu", keep=False,
                 out=None, pre=None):
    """h[t] = act(G_e x[t]) * (U_e x[t]) for the rows t of every expert e.  x: bf16 [rows, in], w:
    bf16 [experts, 2 hidden, in], each expert's gate G_e above its U_e; activation "silu" or
    "gelu" (by the normal distribution function); returns bf16 [rows, hidden].  With keep (or pre to
    write them to) also the products that gated_dgrad needs: (h, pre), pre bf16 [rows, 2 hidden]."""
    E, two, i = _weights("w", w, torch.bfloat16).shape
    if two % 2:
        raise ValueError("w must have a gate row for each of the others")
    _matrix("x", x, torch.bfloat16, i)
    act = _activation(activation)
    _of(E, offsets, mask, x)
    h = _output(out, mask, x.shape[0], two // 2, x)
    if keep or pre is not None:
        pre = _output(pre, mask, x.shape[0], two, x)
    _same_device(x, w, h, pre)
    device, stream = _on(x)
    with device:
        B.gnmr_gated_linear(x, _stride(x), w, pre, 0 if pre is None else _stride(pre), h,
                            _stride(h), x.shape[0], E, two // 2, i, act, offsets, mask, mask_value,
                            stream)
    return h if pre is None else (h, pre)


def gated_activation(pre, offsets=None, mask=None, mask_value=1, activation="silu", out=None):
    """h = act(pre's first half) * (its second half), for products that other operators made.  The
    number of experts is that of offsets."""
    _matrix("pre", pre, torch.bfloat16)
    if pre.shape[1] % 2:
        raise ValueError("pre must have a gate column for each of the others")
    act = _activation(activation)
    E = 1 if offsets is None else offsets.numel() - 1
    _of(E, offsets, mask, pre)
    h = _output(out, mask, pre.shape[0], pre.shape[1] // 2, pre)
    _same_device(pre, h)
    device, stream = _on(pre)
    with device:
        B.gnmr_gated_activation(pre, _stride(pre), h, _stride(h), pre.shape[0], E,
                                pre.shape[1] // 2, act, offsets, mask, mask_value, stream)
    return h


def gated_dgrad(dy, w, pre, offsets=None, mask=None, mask_value=1, activation="silu", out=None):
    """The gradient of gated_linear's products from dy, that of the block's output behind its down
    projection w (bf16 [experts, out, hidden]): (dy W_e) times the derivatives of act(gate) * up at
    pre.  Returns bf16 [rows, 2 hidden]: grouped_dgrad and grouped_wgrad take it on."""
    E, o, hidden = _weights("w", w, torch.bfloat16).shape
    _matrix("dy", dy, torch.bfloat16, o)
    _matrix("pre", pre, torch.bfloat16, 2 * hidden)
    if pre.shape[0] != dy.shape[0]:
        raise ValueError("dy and pre must have the same rows")
    act = _activation(activation)
    _of(E, offsets, mask, dy)
    dpre = _output(out, mask, dy.shape[0], 2 * hidden, dy)
    _same_device(dy, w, pre, dpre)
    device, stream = _on(dy)
    with device:
        B.gnmr_gated_dgrad(dy, _stride(dy), w, pre, _stride(pre), dpre, _stride(dpre),
                           dy.shape[0], E, o, hidden, act, offsets, mask, mask_value, stream)
    return dpre


def _rows_of(t):
    """t's rows over its last dimension, as a matrix whose rows the kernels can read where they lie."""
    flat = t if t.dim() == 2 else t.reshape(-1, t.shape[-1])
    rows, cols = flat.shape
    if (cols > 1 and flat.stride(1) != 1) or (rows > 1 and flat.stride(0) < cols):
        flat = flat.contiguous()
    return flat


def _row_stride(t):
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)


def _vectors(x, cols, **vectors):
    """The type of the weight and bias of layer norm, those that there are."""
    kind = None
    for name, t in vectors.items():
        if t is None:
            continue
        if t.dtype not in _DTYPES or t.shape != (cols,) or t.device != x.device or \
                not t.is_contiguous():
            raise TypeError(f"{name} must be a contiguous bf16 or fp32 tensor of {cols} values on x's "
                            "device")
        if kind not in (None, t.dtype):
            raise TypeError("weight and bias must be of one type")
        kind = t.dtype
    return kind or torch.float32


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None):
    """(y, mean, rstd): layer norm over x's last dimension, y = (x - mean) rstd weight + bias, and
    the fp32 statistics of each row that layer_norm_backward takes.  x: bf16 or fp32, any leading
    dimensions and row strides, 1 to 16384 columns and up to 16,777,215 rows; weight and bias: bf16 or
    fp32, of one type, or None."""
    kind = _DTYPES.get(x.dtype)
    if kind is None or not x.is_cuda or x.dim() < 1:
        raise TypeError("x must be a bf16 or fp32 tensor of rows on a HIP device")
    shape, where = x.shape, x.device
    cols = shape[-1]
    wt = _DTYPES[_vectors(x, cols, weight=weight, bias=bias)]
    flat = _rows_of(x)
    if out is None:
        y = torch.empty_like(x) if flat is x and x.is_contiguous() else torch.empty(
            shape, dtype=x.dtype, device=where)
    else:
        y = out
        if y.shape != shape or y.dtype != x.dtype or y.device != where or \
                (y.dim() != 2 and not y.is_contiguous()) or \
                (y.dim() == 2 and ((cols > 1 and y.stride(1) != 1) or
                                   (y.shape[0] > 1 and y.stride(0) < cols))):
            raise TypeError("out must have x's shape, type and device, and contiguous rows")
    yflat = y if y.dim() == 2 else y.view(-1, cols)
    rows = flat.shape[0]
    mean = torch.empty(rows, dtype=torch.float32, device=where)
    if len(shape) != 2:
        mean = mean.view(shape[:-1])
    rstd = torch.empty_like(mean)
    device, stream = _on(x)
    with device:
        B.gnmr_layer_norm(flat, kind, _row_stride(flat), weight, bias, wt, yflat,
                          _row_stride(yflat), mean, rstd, rows, cols, eps, stream)
    return y, mean, rstd


def layer_norm_backward(dy, x, mean, rstd, weight=None, bias=False, input_grad=True,
                        weight_grad=True):
    """(dx, dweight, dbias) of layer_norm, from dy (of x's type and shape) and what it returned.
    dweight comes with a weight, in its type; dbias where bias is asked for, in that type too, or
    fp32 without a weight; input_grad and weight_grad False leave dx and dweight out (None)."""
    kind = _DTYPES.get(x.dtype)
    if kind is None or not x.is_cuda or x.dim() < 1:
        raise TypeError("x must be a bf16 or fp32 tensor of rows on a HIP device")
    shape, where = x.shape, x.device
    cols = shape[-1]
    if dy.shape != shape:
        raise ValueError(f"dy must have x's shape {tuple(shape)}")
    if dy.dtype != x.dtype:
        raise TypeError(f"dy must be of x's type, {x.dtype}")
    for name, t in (("mean", mean), ("rstd", rstd)):
        if t.dtype != torch.float32 or t.shape != shape[:-1] or not t.is_contiguous():
            raise TypeError(f"{name} must be a contiguous fp32 tensor of an entry per row")
    type_ = _vectors(x, cols, weight=weight)
    _same_device(x, dy, mean, rstd)
    xs, ds = _rows_of(x), _rows_of(dy)
    dx = dw = db = work = None
    if input_grad:
        dx = torch.empty_like(x) if xs is x and x.is_contiguous() else torch.empty(
            shape, dtype=x.dtype, device=where)
    if weight is not None and weight_grad:
        dw = torch.empty_like(weight)
    if bias:
        db = torch.empty(cols, dtype=type_, device=where)
    rows, n = xs.shape[0], 0
    if dw is not None or db is not None:
        n = _norm_workspace(rows, cols)
        if n:
            work = torch.empty(n, dtype=torch.uint8, device=where)
    device, stream = _on(x)
    with device:
        B.gnmr_layer_norm_backward(ds, _row_stride(ds), xs, kind, _row_stride(xs), mean, rstd,
                                   weight, _DTYPES[type_], dx, cols, dw, db, rows, cols, work, n,
                                   stream)
    return dx, dw, db


def clip_gradients(gradients, max_norm, out=None, known=(), norms=None, eps=1e-6):
    """The gradients' global norm (a float64 scalar on their device), and the gradients scaled by
    min(1, max_norm / (norm + eps)): in place, or into `out`, as many bf16 or fp32 tensors of their
    shapes.  gradients: contiguous bf16 or fp32 tensors on one device.  known: indexes of gradients
    whose norms are among `norms` (contiguous float64 on the device; the controller's, for
    instance), so that they need no reading for the global norm.  Where that is at most max_norm, gradients
    in place are not touched."""
    gradients = list(gradients)
    outs = gradients if out is None else list(out)
    count, known = len(gradients), set(known)
    if not gradients:
        raise ValueError("no gradient given")
    if len(outs) != count:
        raise ValueError(f"out must have {count} tensors, not {len(outs)}")
    like = gradients[0]
    device = like.device
    if known:
        if not known.issubset(range(count)):
            raise ValueError("known must be indexes of gradients")
        if norms is None:
            raise ValueError("known gradients need norms")
    if norms is not None and (norms.dtype != torch.float64 or not norms.is_contiguous() or
                              norms.device != device):
        raise TypeError("norms must be a contiguous float64 tensor on the gradients' device")

    def types(name, tensors):
        kinds = [_DTYPES.get(t.dtype) for t in tensors]
        if None in kinds or not all(map(_T.is_contiguous, tensors)) or not like.is_cuda:
            raise TypeError(f"every {name} must be a contiguous bf16 or fp32 tensor on a HIP device")
        if list(map(_T.get_device, tensors)).count(device.index) != count:
            raise ValueError("all gradients must be on one device")
        return kinds
    kinds = out_kinds = types("gradient", gradients)
    if out is not None:
        out_kinds = types("out", outs)
        if any([o.shape != g.shape for g, o in zip(gradients, outs)]):
            raise ValueError("every out must have its gradient's shape")
    table = list(zip(gradients, outs, map(_T.numel, gradients), kinds, out_kinds,
                     [k in known for k in range(count)] if known else [0] * count))
    norm = torch.empty((), dtype=torch.float64, device=device)
    n = _clip_workspace(count)
    work = torch.empty(n, dtype=torch.uint8, device=device)
    context, stream = _on(like)
    with context:
        B.gnmr_clip_gradients(table, max_norm, norm, work, n, norms,
                              0 if norms is None else norms.numel(), eps, stream)
    return norm
