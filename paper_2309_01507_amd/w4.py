"""Layers and a loss over the 4-bit weights' entry points, for models that keep their weights in 4 bits and train what is
left: the groups' scales, or whatever stands in front of the layers.  Orchestration only -- every number is computed by lpmm4.so.

    layer = W4Linear.from_weight(linear.weight, group=128)        # scales are its parameter, codes a buffer
    loss = distill_loss(student(x), top, index, tau=2.0).mean()   # top, index: the teacher's largest logits
    loss.backward(); AdamW4bit([layer.scales]).step()

Inputs are float32 or bfloat16, (..., in_features); gradients of gradients are not defined.
"""
from __future__ import annotations

import torch

from . import binding as _b


def _flat(x: torch.Tensor, cols: int) -> torch.Tensor:
    """(..., cols) as a matrix whose rows' elements are next to each other and do not overlap (an expanded gradient does)"""
    x = x.reshape(-1, cols)
    if x.shape[0] > 1 and (x.stride(0) < cols or x.stride(1) != 1) or x.shape[0] == 1 and cols > 1 and x.stride(1) != 1:
        x = x.contiguous()
    return x


class _Product(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, scales, w):
        flat = _flat(x.detach(), w.cols)
        ctx.rows, ctx.cols, ctx.group, ctx.shape = w.rows, w.cols, w.group, x.shape
        ctx.save_for_backward(flat if ctx.needs_input_grad[1] else None, scales, w.codes)
        return _b.lpmm_w4_linear(flat, w).view(*x.shape[:-1], w.rows)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, scales, codes = ctx.saved_tensors
        w = _b.WeightsW4(ctx.rows, ctx.cols, ctx.group, codes, scales.detach())
        dy = _flat(dy, w.rows)
        dx = _b.lpmm_w4_linear_dx(dy, w).view(ctx.shape) if ctx.needs_input_grad[0] else None
        dscales = _b.lpmm_w4_linear_dscale(x, dy, w) if ctx.needs_input_grad[1] else None
        return dx, dscales, None


def w4_linear(x: torch.Tensor, w: "_b.WeightsW4") -> torch.Tensor:
    """y = x W^T for x (..., cols), with gradients for x and for w.scales."""
    if x.shape[-1] != w.cols:
        raise ValueError(f"w4_linear: the last dimension must be {w.cols}")
    scales = w.scales
    return _Product.apply(x, scales, _b.WeightsW4(w.rows, w.cols, w.group, w.codes, scales.detach()))


class W4Linear(torch.nn.Module):
    """A linear layer without bias whose weight is kept in 4 bits.  `scales` is a parameter (float32, out_features x groups, whatever the
    module is cast to), `codes` a buffer; both are part of the state_dict."""

    def __init__(self, in_features: int, out_features: int, group: int = 128, device="cuda"):
        super().__init__()
        w = _b.new_w4(out_features, in_features, group, device)
        self.in_features, self.out_features, self.group = in_features, out_features, group
        self.register_buffer("codes", w.codes.zero_())
        self.scales = torch.nn.Parameter(w.scales.zero_())

    @classmethod
    def from_weight(cls, weight: torch.Tensor, group: int = 128) -> "W4Linear":
        """weight: out_features x in_features, float32 or bfloat16, on the current GPU"""
        weight = _flat(weight.detach(), weight.shape[-1])
        layer = cls(weight.shape[1], weight.shape[0], group, weight.device)
        _b.lpmm_w4_quant(weight, group, _b.WeightsW4(weight.shape[0], weight.shape[1], group, layer.codes, layer.scales.data))
        return layer

    def _apply(self, fn, recurse=True):
        """Moves between devices are followed; casts (bfloat16(), to(torch.half), ...) leave codes, scales and their gradient as they are."""
        def keep(t):
            moved = fn(t)
            if moved.dtype != t.dtype and (t is self.scales or t is self.scales.grad or t is self.codes):
                moved = t.to(moved.device)
            return moved
        return super()._apply(keep, recurse)

    def weights(self) -> "_b.WeightsW4":
        return _b.WeightsW4(self.out_features, self.in_features, self.group, self.codes, self.scales)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        return w4_linear(x, self.weights())

    def extra_repr(self) -> str:
        return f"in_features={self.in_features}, out_features={self.out_features}, group={self.group}"


class _Distill(torch.autograd.Function):
    @staticmethod
    def forward(ctx, z, top, index, tau):
        loss, lse = _b.lpmm_distill_loss(z.detach(), top, index, tau)
        ctx.tau = tau
        ctx.save_for_backward(z, top, index, lse)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        z, top, index, lse = ctx.saved_tensors
        return _b.lpmm_distill_grad(z.detach(), top, index, ctx.tau, lse, grad.contiguous()), None, None, None


def distill_loss(logits: torch.Tensor, top: torch.Tensor, index: torch.Tensor, tau: float = 1.0) -> torch.Tensor:
    """Loss of each token against a teacher's largest logits (lpmm_distill_loss): logits (..., vocabulary), top and index (..., slots),
    index -1 in slots that do not count; the result has the leading dimensions.  The teacher gets no gradient: detach its logits."""
    if top.requires_grad and torch.is_grad_enabled():
        raise ValueError("distill_loss: there is no gradient for the teacher's logits; detach them")
    lead = logits.shape[:-1]
    if top.shape[:-1] != lead or index.shape != top.shape:
        raise ValueError(f"distill_loss: top and index must be {tuple(lead)} x slots, like the logits")
    z = _flat(logits, logits.shape[-1])
    loss = _Distill.apply(z, top.reshape(-1, top.shape[-1]).contiguous(), index.reshape(-1, index.shape[-1]).contiguous(), float(tau))
    return loss.view(lead)
