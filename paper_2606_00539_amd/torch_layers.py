"""Layers on libgnmr's operators, recorded by autograd.

Argument marshalling only: the kernels run in libgnmr, on torch's current stream of the
tensors' device.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import torch_ops as ops


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = ops.layer_norm(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.bias_type = None if bias is None else bias.dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        of_x, of_weight, of_bias, _ = ctx.needs_input_grad
        dx, dw, db = ops.layer_norm_backward(dy, x, mean, rstd, weight, bias=of_bias,
                                             input_grad=of_x, weight_grad=of_weight)
        return dx, dw, None if db is None else db.to(ctx.bias_type), None


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over x's last dimension (K10), with the gradients of x, weight and bias.  x: bf16
    or fp32 on a HIP device, 1 to 16384 columns, up to 16,777,215 rows; weight and bias: bf16 or fp32,
    both of one type.  Second derivatives are refused.  As with torch's own operators, backward is
    captured in a graph only while no autograd graph made outside the capture holds the same leaves."""
    return _LayerNorm.apply(x, weight, bias, eps)


class LayerNorm(torch.nn.Module):
    """Layer norm over the last dimension, of `dim` values, with a weight and a bias to learn."""

    def __init__(self, dim: int, eps: float = 1e-5, bias: bool = True, device="cuda",
                 dtype=torch.float32):
        super().__init__()
        if not 1 <= dim <= 16384:
            raise ValueError(f"dim must be in [1, 16384], got {dim}")
        if dtype not in (torch.bfloat16, torch.float32):
            raise TypeError("dtype must be torch.bfloat16 or torch.float32")
        self.dim, self.eps = int(dim), float(eps)
        self.weight = torch.nn.Parameter(torch.ones(dim, device=device, dtype=dtype))
        self.register_parameter("bias", torch.nn.Parameter(
            torch.zeros(dim, device=device, dtype=dtype)) if bias else None)

    def forward(self, x):
        return layer_norm(x, self.weight, self.bias, self.eps)

    def extra_repr(self):
        return f"{self.dim}, eps={self.eps}, bias={self.bias is not None}"
