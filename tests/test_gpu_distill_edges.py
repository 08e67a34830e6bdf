"""Distillation's gradient where a row's lse says little: large logits, and rows of nothing but a mask's lowest value."""
import pytest
import torch

import paper_2309_01507_amd as lpmm
import w4_util as ref
from conftest import progress
from w4_util import DEV

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("v", [40, 1031, 9001, 140001])
def test_gradient_of_large_and_of_masked_rows(v, tau, dtype):
    """The softmax in 64 bits from differences to the row's maximum, which are exact.  A kernel's exponent errs by a few units of 2^-24 of that difference,
    or, while lse is below 1024, of its own two parts; sums as in the other tests."""
    progress(f"distill large rows of {v}, tau {tau} {dtype}")
    g = torch.Generator().manual_seed(v)
    z = 2.0 * torch.randn(8, v, generator=g)
    z[1] += 3.0e4
    z[2] -= 700.0 * tau
    z[3] = torch.finfo(dtype).min
    z[4] = torch.finfo(dtype).min
    z[4, v // 2:] = -float("inf")
    z[5] = 1.0e37
    z[6, : v // 2] = torch.finfo(dtype).min
    z = z.to(dtype)
    slots = 9
    top, index = torch.randn(8, slots, generator=g), torch.randint(0, v // 2, (8, slots), generator=g)
    index[:, 4] = index[:, 2]
    grad = torch.rand(8, generator=g)
    x = z.double() / tau
    away = x - x.amax(dim=1, keepdim=True)
    q = torch.softmax(away, dim=1)
    p = torch.softmax(top.double() / tau, dim=1)
    target = torch.zeros(8, v).double().scatter_add_(1, index, p)
    want = grad.double()[:, None] * tau * (q - target)
    lse = x.amax(dim=1, keepdim=True) + torch.log(torch.exp(away).sum(dim=1, keepdim=True))
    part = torch.where(lse.abs() < 1025, lse.abs() + x.abs().clamp(max=2000), torch.zeros_like(lse))
    u = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    err = 2.0 ** -24 * (q * (64 + 4 * away.abs().clamp(max=2000) + 2 * part) + target * (64 + 4 * top.abs().amax(dim=1, keepdim=True) / tau))
    tol = u * want.abs() + (1 + u) * grad.double()[:, None] * tau * err + 1e-37
    zd, td, xd, gd = z.to(DEV), top.to(DEV), index.to(DEV), grad.to(DEV)
    _, got_lse = lpmm.lpmm_distill_loss(zd, td, xd, tau)
    ref.assert_within(lpmm.lpmm_distill_grad(zd, td, xd, tau, got_lse, gd), want, tol, "two calls")
    ref.assert_within(lpmm.lpmm_distill_loss_grad(zd, td, xd, tau, gd)[1], want, tol, "one call")
    ref.assert_within(lpmm.lpmm_distill_grad(zd, td, xd, tau, got_lse, gd, zd), want, tol, "in place")


@pytest.mark.parametrize("t,v,dtype", [(3600, 33001, BF16), (3500, 51200, BF16), (3, 20001, F32), (1100, 25600, F32), (3, 60001, F32), (3600, 17000, F32), (5, 51201, BF16)])
def test_rows_in_registers_of_every_shape(t, v, dtype):
    """Loss and gradient at once, against 64 bits on the GPU; bounds as in the other tests."""
    progress(f"distill at once {t} x {v} {dtype}")
    g = torch.Generator(device=DEV).manual_seed(t)
    slots, tau = 6, 1.5
    z = (2.5 * torch.randn(t, v, generator=g, device=DEV)).to(dtype)
    top, index = 4.0 + torch.randn(t, slots, generator=g, device=DEV), torch.randint(0, v, (t, slots), generator=g, device=DEV)
    grad = torch.rand(t, generator=g, device=DEV)
    loss, dz = lpmm.lpmm_distill_loss_grad(z, top, index, tau, grad)
    u = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24
    for first in range(0, t, 512):
        r = slice(first, min(first + 512, t))
        x = z[r].double() / tau
        log_q = torch.log_softmax(x, dim=1)
        p = torch.softmax(top[r].double() / tau, dim=1)
        at = log_q.gather(1, index[r])
        want_loss = tau * tau * (p * (p.log() - at)).sum(dim=1)
        size = (p * (at.abs() + 2 * top[r].double().abs() / tau + 16)).sum(dim=1)
        q = log_q.exp()
        target = torch.zeros_like(q).scatter_add_(1, index[r], p)
        want = grad[r].double()[:, None] * tau * (q - target)
        err = 2.0 ** -24 * (q * (64 + 4 * x.abs() + 4 * log_q.abs()) + target * (64 + 4 * top[r].double().abs().amax(dim=1, keepdim=True) / tau))
        tol = u * want.abs() + (1 + u) * grad[r].double()[:, None] * tau * err + 1e-37
        over = (dz[r].double() - want).abs() - tol
        assert float(over.max()) <= 0, f"dz: {int((over > 0).sum())} too far off, worst by {float(over.max()):.3g}"
        over = (loss[r].double() - want_loss).abs() - (tau * tau * 2.0 ** -24 * (8 * size + 80) + 2.0 ** -22 * want_loss.abs())
        assert float(over.max()) <= 0, f"loss: worst by {float(over.max()):.3g}"
