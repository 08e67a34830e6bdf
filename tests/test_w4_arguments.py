"""What the 4-bit weights' and distillation's calls refuse before they touch a GPU, and what the layer does with a cast: no GPU needed."""
import pytest
import torch

import paper_2309_01507_amd as lpmm

ROWS, COLS, GROUP = 48, 160, 32


def on_cpu(codes=torch.uint8, scales=torch.float32):
    room = lpmm.lpmm_w4_sizes(ROWS, COLS, GROUP)
    return lpmm.WeightsW4(ROWS, COLS, GROUP, torch.zeros(room[0], dtype=codes), torch.zeros(ROWS, room[1] // 4 // ROWS, dtype=scales))


@pytest.mark.parametrize("codes,scales", [(torch.uint8, torch.bfloat16), (torch.uint8, torch.float16), (torch.uint8, torch.float64),
                                          (torch.int8, torch.float32), (torch.int32, torch.float32)])
def test_codes_and_scales_of_another_type(codes, scales):
    """Scales of two bytes each would be read, and by the compressing call written, beyond their end."""
    w = on_cpu(codes, scales)
    x, dy = torch.zeros(3, COLS), torch.zeros(3, ROWS)
    for call in (lambda: lpmm.lpmm_w4_linear(x, w), lambda: lpmm.lpmm_w4_linear_dx(dy, w), lambda: lpmm.lpmm_w4_linear_dscale(x, dy, w),
                 lambda: lpmm.lpmm_w4_dequant(w), lambda: lpmm.lpmm_w4_quant(torch.zeros(ROWS, COLS), GROUP, w), lambda: lpmm.w4_linear(x, w)):
        with pytest.raises(ValueError, match="codes must be uint8 and scales float32"):
            call()


@pytest.mark.parametrize("cast", [lambda m: m.bfloat16(), lambda m: m.half(), lambda m: m.double(), lambda m: m.to(torch.bfloat16),
                                  lambda m: m.to("cpu", torch.float16), lambda m: m.type(torch.bfloat16), lambda m: m.float()])
def test_a_cast_leaves_the_scales_as_they_are(cast):
    layer = lpmm.W4Linear(COLS, ROWS, GROUP, device="cpu")
    torch.nn.init.uniform_(layer.scales, 0.01, 0.02)
    layer.codes.random_(0, 256)
    scales, codes, parameter = layer.scales.detach().clone(), layer.codes.clone(), layer.scales
    parameter.grad = torch.rand_like(scales)
    grad = parameter.grad.clone()
    model = torch.nn.Sequential(layer, torch.nn.Linear(ROWS, 4), torch.nn.LayerNorm(4))
    cast(model)
    assert layer.scales is parameter and parameter.requires_grad and torch.equal(parameter.detach(), scales)
    assert parameter.dtype == parameter.grad.dtype == torch.float32 and torch.equal(parameter.grad, grad)
    assert layer.codes.dtype == torch.uint8 and torch.equal(layer.codes, codes)
    other = cast(torch.nn.Linear(2, 2))
    assert model[1].weight.dtype == model[2].weight.dtype == other.weight.dtype, "the cast still holds for the rest of the model"
    assert layer.to("meta").scales.device.type == "meta"


@pytest.mark.parametrize("workspace", [torch.empty(1).expand(1 << 20), torch.empty(2, 64).t()])
def test_a_workspace_with_gaps_or_repeats(workspace):
    """An expanded tensor has fewer bytes than elements."""
    from paper_2309_01507_amd import binding
    with pytest.raises(ValueError, match="contiguous"):
        binding._workspace(workspace, 64, torch.empty(1), None, "call")
    whole = torch.empty(64)
    assert binding._workspace(whole, 64, torch.empty(1), None, "call") is whole


@pytest.mark.parametrize("tau,fine", [(3.5e-39, False), (4.2e-39, False), (4.5e-39, True), (1e-3, True), (1.0, True), (1.8e19, True), (1.9e19, False),
                                      (3.0e38, False), (float("inf"), False), (float("nan"), False), (0.0, False), (-1.0, False)])
def test_temperatures_beyond_fp32(tau, fine):
    """log2(e) / tau or tau^2 of infinity would meet a difference of 0.  No rows: nothing is launched."""
    L = lpmm.lib()
    want = 0 if fine else -1
    args = [None, 0, 0, 100, 100, None, None, 6, tau]
    assert L.lpmm_distill_loss(*args, None, None, None, 0, None) == want
    assert L.lpmm_distill_grad(*args, None, None, None, 100, None) == want
    assert L.lpmm_distill_loss_grad(*args, None, None, None, None, 100, None, 0, None) == want


def test_a_teacher_that_wants_a_gradient():
    z, top, index = torch.zeros(2, 10, requires_grad=True), torch.zeros(2, 3, requires_grad=True), torch.zeros(2, 3, dtype=torch.int64)
    with pytest.raises(ValueError, match="detach"):
        lpmm.distill_loss(z, top, index)
    for call in (lambda: lpmm.distill_loss(z, top.detach(), index), lambda: torch.no_grad()(lpmm.distill_loss)(z, top, index)):
        with pytest.raises(ValueError, match="on the current GPU"):            # no GPU here: the next thing that is refused
            call()


@pytest.mark.parametrize("shape", [(3, 2, 4), (6, 4), (2, 2, 4), (4,)])
def test_a_teacher_of_another_shape(shape):
    """As many rows in another order would be paired with the wrong tokens."""
    z, top, index = torch.zeros(2, 3, 10), torch.zeros(2, 3, 4), torch.zeros(2, 3, 4, dtype=torch.int64)
    for a, b in ((torch.zeros(shape), torch.zeros(shape, dtype=torch.int64)), (torch.zeros(shape), index), (top, torch.zeros(shape, dtype=torch.int64))):
        with pytest.raises(ValueError, match="like the logits"):
            lpmm.distill_loss(z, a, b)
