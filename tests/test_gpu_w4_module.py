"""The layers over the 4-bit weights, and everything together: a student in 4 bits trained on its teacher's top logits."""
import pytest
import torch

import paper_2309_01507_amd as lpmm
import w4_util as ref
from w4_util import DEV

pytestmark = pytest.mark.gpu


def test_layer_gradients_through_autograd():
    """(2, 3, in) inputs, a gradient that arrives expanded and one that arrives transposed; against plain 64-bit autograd."""
    torch.manual_seed(3)
    layer = lpmm.W4Linear.from_weight(torch.randn(48, 160, device=DEV), 32)
    q = ref.unpack(layer.codes, 48, 160)
    x = torch.randn(2, 3, 160, device=DEV, requires_grad=True)
    x64 = x.detach().cpu().double().requires_grad_()
    s64 = layer.scales.detach().cpu().double().requires_grad_()
    y64 = x64 @ (ref.VALUES[q] * s64.repeat_interleave(32, dim=1)).t()
    for what in ("expanded", "transposed"):
        for p in (x, layer.scales, x64, s64):
            p.grad = None
        y = layer(x)
        if what == "expanded":
            y.sum().backward()
            y64.sum().backward(retain_graph=True)
        else:
            c = torch.randn(48, 3, 2, device=DEV)
            (y * c.permute(2, 1, 0)).sum().backward()
            (y64 * c.cpu().double().permute(2, 1, 0)).sum().backward(retain_graph=True)
        # fp32 sums of 160, 48 and 6 + 32 terms: errors of a few units of 2^-24 of the terms' sizes, far below 1e-5 of the largest
        assert float((y.detach().cpu().double() - y64.detach()).abs().max()) < 1e-5 * float(y64.abs().max())
        assert float((x.grad.cpu().double() - x64.grad).abs().max()) < 1e-5 * float(x64.grad.abs().max())
        assert float((layer.scales.grad.cpu().double() - s64.grad).abs().max()) < 1e-5 * float(s64.grad.abs().max())


def test_layer_state_and_frozen_parts():
    torch.manual_seed(4)
    layer = lpmm.W4Linear.from_weight(torch.randn(33, 100, device=DEV).bfloat16(), 64)
    other = lpmm.W4Linear(100, 33, 64)
    other.load_state_dict(layer.state_dict())
    x = torch.randn(5, 100, device=DEV)
    assert torch.equal(layer(x), other(x))
    layer.scales.requires_grad_(False)
    x.requires_grad_()
    layer(x).sum().backward()
    assert layer.scales.grad is None and x.grad is not None
    y = layer(x.detach())
    assert not y.requires_grad
    assert layer(torch.empty(0, 100, device=DEV)).shape == (0, 33)
    with pytest.raises(ValueError):
        layer(torch.randn(5, 99, device=DEV))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_loss_through_autograd(dtype):
    g = torch.Generator().manual_seed(2)
    z = (2 * torch.randn(2, 4, 300, generator=g)).to(dtype)
    top, index = torch.randn(2, 4, 5, generator=g), torch.randint(0, 300, (2, 4, 5), generator=g)
    index[0, 1] = -1
    zd = z.to(DEV).requires_grad_()
    loss = lpmm.distill_loss(zd, top.to(DEV), index.to(DEV), 2.0)
    assert loss.shape == (2, 4) and float(loss[0, 1]) == 0.0
    (loss * torch.arange(8, device=DEV).view(2, 4)).sum().backward()
    want_loss, _, want = ref.distill(z.view(8, 300), top.view(8, 5), index.view(8, 5), 2.0, torch.arange(8.0))
    assert float((loss.detach().cpu().double().view(8) - want_loss).abs().max()) < 1e-5 * float(want_loss.max())
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -20
    got = zd.grad.cpu().double().view(8, 300)
    assert bool(((got - want).abs() <= u * want.abs() + 1e-5).all())
    logits = zd.transpose(0, 1)                          # rows that are not next to each other in order
    again = lpmm.distill_loss(logits, top.to(DEV).transpose(0, 1), index.to(DEV).transpose(0, 1), 2.0)
    assert torch.equal(again.transpose(0, 1), loss.detach())


def test_recovery():
    """Training the scales on the teacher's top logits lowers the loss on text that was not trained on, and a token at a time
    the student says what it says to the whole text."""
    from paper_2309_01507_amd import w4_recovery
    before, after, off = w4_recovery.recover(60)
    print(f"[gpu-test] recovery {before:.5f} -> {after:.5f}, token by token off by {off:.1e}", flush=True)
    assert after < 0.9 * before
    assert off < 1e-4


def test_a_cast_layer_computes_in_bf16():
    """After model.to(torch.bfloat16) the layer takes bf16 inputs and its scales are the ones it had."""
    torch.manual_seed(5)
    layer = lpmm.W4Linear.from_weight(torch.randn(96, 200, device=DEV), 64)
    full = ref.VALUES[ref.unpack(layer.codes, 96, 200)] * ref.spread(layer.scales.detach().cpu(), 64, 200)
    model = torch.nn.Sequential(layer).to(torch.bfloat16)
    x = torch.randn(7, 200, device=DEV).bfloat16().requires_grad_()
    y = model(x)
    y.backward(torch.ones_like(y))
    want, mag = x.detach().cpu().double() @ full.t(), x.detach().cpu().double().abs() @ full.abs().t()
    ref.assert_within(y.detach(), want, ref.bound(torch.bfloat16, want, mag, 204), "y")
    assert layer.scales.grad.dtype == torch.float32 and x.grad.dtype == torch.bfloat16


@pytest.mark.parametrize("part", ["codes", "scales", "both"])
def test_weights_quantized_anew_between_forward_and_backward(part):
    """The gradient would be that of other weights than the product's."""
    torch.manual_seed(6)
    layer = lpmm.W4Linear.from_weight(torch.randn(40, 96, device=DEV), 32)
    x = torch.randn(3, 96, device=DEV, requires_grad=True)
    y = layer(x)
    if part == "codes":
        layer.codes.copy_(layer.codes.flip(0))
    elif part == "scales":
        with torch.no_grad():
            layer.scales.mul_(2)
    else:
        lpmm.lpmm_w4_quant(torch.randn(40, 96, device=DEV), 32, layer.weights())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    layer(x).sum().backward()
    assert x.grad is not None and layer.scales.grad is not None
    with torch.inference_mode():
        lpmm.lpmm_w4_quant(torch.randn(40, 96, device=DEV), 32, lpmm.new_w4(40, 96, 32))


def test_logits_overwritten_by_their_gradient_between_forward_and_backward():
    """dz may be z; a backward pass that still needs the logits says so."""
    z = torch.randn(4, 50, device=DEV, requires_grad=True)
    logits = z * 1.0
    top, index, grad = torch.randn(4, 3, device=DEV), torch.randint(0, 50, (4, 3), device=DEV), torch.ones(4, device=DEV)
    for overwrite in (lambda: lpmm.lpmm_distill_loss_grad(logits.detach(), top, index, 1.0, grad, dz=logits.detach()),
                      lambda: lpmm.lpmm_distill_grad(logits.detach(), top, index, 1.0, torch.zeros(4, device=DEV), grad, logits.detach())):
        loss = lpmm.distill_loss(logits, top, index).sum()
        overwrite()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward(retain_graph=True)
    lpmm.distill_loss(logits, top, index).sum().backward()
