"""A linear layer whose products, forward and backward, are of 8-bit operands with a power of two for each block of 128.
Orchestration only -- every number is computed by lpmm4.so.

    layer = F8Linear(in_features, out_features)                   # weight: a float32 parameter
    y = layer(x); y.backward(dy); AdamW4bit([layer.weight]).step()

    y  = Q(x) Q(W)^T          x and dy in blocks of 1 x 128 along the sum, W in blocks of 128 x 128
    dx = Q(dy) Q(W)
    dW = Q(dy^T) Q(x^T)^T     blocks of 1 x 128 along the tokens

Rounding to 8 bits passes gradients through as they are.  Inputs are float32 or bfloat16, (..., in_features); gradients of gradients are
not defined.  Weights that stay as they are can be kept in 8 bits alone: lpmm_f8_quant(weight, 128) once, then lpmm_f8_linear.
"""
from __future__ import annotations

import torch

from . import binding as _b
from .w4 import _flat


class _Product(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight):
        flat = _flat(x.detach(), weight.shape[1])
        w = weight.detach()
        t = flat.shape[0]
        need_x, need_w = ctx.needs_input_grad
        qw, qwt = _b.lpmm_f8_quant_both(w, 128) if need_x else (_b.lpmm_f8_quant(w, 128), None)
        qxt = None
        if need_w and t:
            qx, qxt = _b.lpmm_f8_quant_both(flat, 1)
            y = _b.lpmm_f8_matmul(qx, qw, flat.dtype)
        else:
            y = _b.lpmm_f8_linear(flat, qw)
        ctx.t, ctx.shape, ctx.w_shape, ctx.w_dtype = t, x.shape, weight.shape, weight.dtype
        ctx.save_for_backward(*((qwt.codes, qwt.scales) if qwt else (None, None)), *((qxt.codes, qxt.scales) if qxt else (None, None)))
        return y.view(*x.shape[:-1], weight.shape[0])

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        w_codes, w_scales, x_codes, x_scales = ctx.saved_tensors
        (n, k), t = ctx.w_shape, ctx.t
        dy = _flat(dy, n)
        dx = dw = None
        need_x, need_w = ctx.needs_input_grad
        if t == 0:
            return (dy.new_zeros(ctx.shape) if need_x else None, dy.new_zeros(n, k, dtype=ctx.w_dtype) if need_w else None)
        if need_w:
            q, qt = _b.lpmm_f8_quant_both(dy, 1)
            dw = _b.lpmm_f8_matmul(qt, _b.MatF8(k, t, 1, x_codes, x_scales), ctx.w_dtype)
            if need_x:
                dx = _b.lpmm_f8_matmul(q, _b.MatF8(k, n, 128, w_codes, w_scales), dy.dtype)
        elif need_x:
            dx = _b.lpmm_f8_linear(dy, _b.MatF8(k, n, 128, w_codes, w_scales))
        return dx.view(ctx.shape) if need_x else None, dw


def f8_linear(x: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
    """y = x W^T by 8-bit products, with gradients for x (..., in_features) and weight (out_features, in_features); float32 or bfloat16 each."""
    if weight.dim() != 2 or x.shape[-1:] != weight.shape[1:]:
        raise ValueError(f"f8_linear: {tuple(x.shape)} and a weight of {tuple(weight.shape)}")
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
