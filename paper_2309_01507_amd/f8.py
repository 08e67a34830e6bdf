"""A linear layer whose products, forward and backward, are of 8-bit operands with a power of two for each block of 128.
Orchestration only -- every number is computed by lpmm4.so.

    layer = F8Linear(in_features, out_features)                   # weight: a float32 parameter
    y = layer(x); y.backward(dy); AdamW4bit([layer.weight]).step()

    y  = Q(x) Q(W)^T          x and dy in blocks of 1 x 128 along the sum, W in blocks of 128 x 128
    dx = Q(dy) Q(W)
    dW = Q(dy^T) Q(x^T)^T     blocks of 1 x 128 along the tokens

Rounding to 8 bits passes gradients through as they are.  Inputs are float32 or bfloat16, (..., in_features); gradients of gradients are
not defined.  A step that is captured into a graph calls lpmm_f8_train_forward and lpmm_f8_train_backward themselves: autograd runs the sum into a leaf's .grad on the
stream that first used the leaf.  Weights that stay as they are can be kept in 8 bits alone: lpmm_f8_quant(weight, 128) once, then lpmm_f8_linear.
"""
from __future__ import annotations

import torch

from . import binding as _b
from .w4 import _flat


class _Product(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight):
        need_x, need_w = ctx.needs_input_grad
        n, k = weight.shape
        flat = _flat(x.detach(), k)
        ctx.grads, ctx.shape, ctx.w_shape, ctx.w_dtype = need_x * _b.F8_DX | need_w * _b.F8_DW, x.shape, weight.shape, weight.dtype
        if flat.shape[0] == 0:
            kept, y = None, flat.new_empty(0, n)
        elif ctx.grads:
            y, kept = _b.lpmm_f8_train_forward(flat, _flat(weight.detach(), k), ctx.grads)
        else:
            kept, y = None, _b.lpmm_f8_linear(flat, _b.lpmm_f8_quant(_flat(weight.detach(), k), 128))
        ctx.save_for_backward(kept)
        return y.view(*x.shape[:-1], n)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        kept, = ctx.saved_tensors
        n, k = ctx.w_shape
        dy = _flat(dy, n)
        if dy.shape[0] == 0:
            return (dy.new_empty(ctx.shape) if ctx.grads & _b.F8_DX else None, dy.new_zeros(n, k, dtype=ctx.w_dtype) if ctx.grads & _b.F8_DW else None)
        dx, dw = _b.lpmm_f8_train_backward(dy, kept, k, ctx.w_dtype, ctx.grads)
        return None if dx is None else dx.view(ctx.shape), dw


def f8_linear(x: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
    """y = x W^T by 8-bit products, with gradients for x (..., in_features) and weight (out_features, in_features); float32 or bfloat16 each."""
    if weight.dim() != 2 or x.shape[-1:] != weight.shape[1:]:
        raise ValueError(f"f8_linear: {tuple(x.shape)} and a weight of {tuple(weight.shape)}")
    if not torch.is_grad_enabled():
        x, weight = x.detach(), weight.detach()              # nothing is laid out for gradients
    return _Product.apply(x, weight)


class F8Linear(torch.nn.Module):
    """A linear layer without bias that computes with 8-bit operands; its weight is an ordinary parameter."""

    def __init__(self, in_features: int, out_features: int, device="cuda", dtype=torch.float32):
        super().__init__()
        self.in_features, self.out_features = in_features, out_features
        self.weight = torch.nn.Parameter(torch.empty(out_features, in_features, device=device, dtype=dtype))
        torch.nn.init.kaiming_uniform_(self.weight, a=5 ** 0.5)

    @classmethod
    def from_weight(cls, weight: torch.Tensor) -> "F8Linear":
        """A copy of weight: out_features x in_features, float32 or bfloat16"""
        layer = cls.__new__(cls)
        torch.nn.Module.__init__(layer)
        layer.out_features, layer.in_features = weight.shape
        layer.weight = torch.nn.Parameter(weight.detach().clone(memory_format=torch.contiguous_format))
        return layer

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return f8_linear(x, self.weight)

    def extra_repr(self) -> str:
        return f"in_features={self.in_features}, out_features={self.out_features}"
