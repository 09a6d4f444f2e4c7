"""The expert step's operators on PyTorch tensors.

  grouped_linear, grouped_dgrad, grouped_wgrad   products grouped by expert
  quantize_rows, quantized_linear                the INT8 low-cost path
  orthogonalize                                  the Newton-Schulz update

Rows (tokens) lie sorted by expert: expert e has rows [offsets[e], offsets[e + 1])
of int32 device `offsets`; rows from offsets[-1] on belong to nobody and give 0.
With `mask` (device bytes or bools, one per expert) only experts whose entry is
`mask_value` are computed, and the outputs of the others stay as they were, so
such a call takes the tensor to write to.

Argument marshalling only: everything runs in libgnmr, on torch's current stream
of the tensors' device.  Nothing here is recorded by autograd (ExpertUnits.linear
in torch_experts.py is).
"""
from __future__ import annotations

import functools

import torch

from . import binding as B

_DTYPES = {torch.bfloat16: B.GNMR_BF16, torch.float32: B.GNMR_F32}
_num_partials = functools.lru_cache(None)(B.gnmr_grouped_wgrad_num_partials)
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
