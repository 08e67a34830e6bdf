"""What sampling, the gradients' norm and clipping refuse before they touch a GPU: no GPU needed."""
import ctypes

import pytest
import torch

import paper_2309_01507_amd as lpmm
from paper_2309_01507_amd import binding as B

NAN, INF = float("nan"), float("inf")


def test_sampling_refuses():
    z, u = torch.zeros(3, 10), torch.zeros(3)
    for bad in (lambda: lpmm.lpmm_sample(z.half(), u), lambda: lpmm.lpmm_sample(z[0], u), lambda: lpmm.lpmm_sample(z.t(), torch.zeros(10)),
                lambda: lpmm.lpmm_sample(z, u[:2]), lambda: lpmm.lpmm_sample(z, u.double()), lambda: lpmm.lpmm_sample(z, torch.zeros(6)[::2]),
                lambda: lpmm.lpmm_sample(z, u, temperature=torch.zeros(2)), lambda: lpmm.lpmm_sample(z, u, top_k=torch.zeros(3)),
                lambda: lpmm.lpmm_sample(z, u, top_p=torch.zeros(3, dtype=torch.bfloat16)), lambda: lpmm.lpmm_sample(z, u, min_p=torch.zeros(6)[::2]),
                lambda: lpmm.lpmm_sample(z, u, tokens=torch.zeros(3, dtype=torch.int32)), lambda: lpmm.lpmm_sample(z, u, logprob=torch.zeros(2)),
                lambda: lpmm.lpmm_sample(z.expand(3, 3, 10), u), lambda: lpmm.lpmm_sample(z[:1].expand(3, 10), u),
                lambda: lpmm.lpmm_sample(z, u, stream=5), lambda: lpmm.lpmm_sample(z, u)):                # the last: not on a GPU
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("name,value,fine", [("temperature", 0.0, True), ("temperature", INF, True), ("temperature", -0.5, False), ("temperature", NAN, False),
                                             ("top_k", 0, True), ("top_k", 2 ** 31 - 1, True), ("top_k", -1, False), ("top_p", NAN, False),
                                             ("top_p", -1.0, True), ("top_p", 2.0, True), ("min_p", NAN, False), ("min_p", 3.0, True)])
def test_options_for_all_rows(name, value, fine):
    """No rows: nothing is launched."""
    o = B.SampleOptions(1.0, 1.0, 0.0, 0)
    setattr(o, name, value)
    assert lpmm.lib().lpmm_sample(None, 0, 0, 100, 100, None, ctypes.addressof(o), None, None, None, 0, None) == (0 if fine else -1)


def test_sampling_sizes():
    o = B.SampleOptions(1.0, 1.0, 0.0, 0)
    call = lambda t, v, ld, dtype=0: lpmm.lib().lpmm_sample(None, dtype, t, v, ld, None, ctypes.addressof(o), None, None, None, 0, None)
    assert call(0, 1, 1) == 0 and call(0, 2 ** 30, 2 ** 30, 1) == 0
    assert call(-1, 1, 1) == call(0, 0, 1) == call(0, 2 ** 30 + 1, 2 ** 31) == call(0, 10, 9) == call(0, 10, 10, 2) == call(2 ** 24, 1, 1) == -1
    assert call(1, 10, 10) == -1, "null pointers"
    assert lpmm.lib().lpmm_sample(None, 0, 0, 1, 1, None, None, None, None, None, 0, None) == -1
    o.temperatures = 2
    assert call(0, 1, 1) == -1, "an array off its boundary"


def descs(*tensors):
    out = (B.GradDesc * max(1, len(tensors)))()
    for i, t in enumerate(tensors):
        out[i] = B.GradDesc(*t)
    return out


def build(device=256, room=None, **given):
    """Refused before anything is copied"""
    d = descs(*given["list"])
    n = len(given["list"])
    need = lpmm.lib().lpmm_grad_plan_bytes(ctypes.addressof(d), n)
    return lpmm.lib().lpmm_grad_plan_build(ctypes.addressof(d), n, device, need if room is None else room, None, ctypes.addressof(B.GradPlanHost()))


def test_plan_sizes():
    size = lambda *t, n=None: lpmm.lib().lpmm_grad_plan_bytes(ctypes.addressof(descs(*t)), len(t) if n is None else n)
    assert size() > 0
    assert size((0, 0, 10, 0, 0)) > size()
    assert size((0, 0, 1 << 33, 1, 0)) > 8 * (1 << 18), "a chunk for each 64 KiB"
    assert size((0, 0, -1, 0, 0)) == size((0, 0, 1, 2, 0)) == size((0, 0, 1, 0, 1)) == size((0, 0, (1 << 40) + 1, 0, 0)) == size(n=-1) == 0
    assert lpmm.lib().lpmm_grad_plan_bytes(None, 1) == 0 and lpmm.lib().lpmm_grad_plan_bytes(None, 0) == size()


def test_plans_without_room():
    one = [(4096, 4096, 10, 0, 0)]
    assert build(list=one, device=None) == build(list=one, device=128) == -1
    assert build(list=one, room=100) == -4


def test_norm_and_clip_arguments():
    L = lpmm.lib()
    norm = 4096
    ok = lambda **k: B.GradPlanHost(**{**dict(device=256, tensors=1, chunks=0, log_bytes=12, writes=1), **k})
    for bad in (ok(device=None), ok(device=128), ok(tensors=-1), ok(chunks=-1), ok(chunks=1 << 31), ok(log_bytes=11), ok(log_bytes=17)):
        assert L.lpmm_grad_norm(ctypes.addressof(bad), 0, norm, None) == -1
        assert L.lpmm_grad_clip(ctypes.addressof(bad), norm, 1.0, None) == -1
    fine = ok()
    assert L.lpmm_grad_norm(None, 0, norm, None) == L.lpmm_grad_norm(ctypes.addressof(fine), 2, norm, None) == -1
    assert L.lpmm_grad_norm(ctypes.addressof(fine), 0, None, None) == L.lpmm_grad_norm(ctypes.addressof(fine), 0, 4098, None) == -1
    for limit in (-1.0, NAN):
        assert L.lpmm_grad_clip(ctypes.addressof(fine), norm, limit, None) == -1
        assert L.lpmm_grad_norm_clip(ctypes.addressof(fine), 0, limit, norm, None) == -1
    for limit in (0.0, 1.0, INF):                                          # no chunks: nothing is launched
        assert L.lpmm_grad_clip(ctypes.addressof(fine), norm, limit, None) == 0
    only_measured = ok(writes=0)
    assert L.lpmm_grad_clip(ctypes.addressof(only_measured), norm, 1.0, None) == -1


def test_lists_of_other_tensors():
    g = torch.zeros(4)
    for bad in (lambda: lpmm.new_grad_plan([g]), lambda: lpmm.new_grad_plan([g.half()]), lambda: lpmm.new_grad_plan([torch.zeros(4, 4).t()]),
                lambda: lpmm.new_grad_plan([g], []), lambda: lpmm.new_grad_plan([g], [torch.zeros(5)])):
        with pytest.raises(ValueError):
            bad()


def test_modules_refuse():
    z = torch.zeros(2, 3, 10)
    for bad in (lambda: lpmm.sample(z, u=torch.zeros(3, 2)), lambda: lpmm.sample(z, temperature=torch.zeros(6)), lambda: lpmm.sample(z, top_k=torch.zeros(2, 3)),
                lambda: lpmm.sample(z), lambda: lpmm.clip_grad_norm([], 1.0, norm_type=1), lambda: lpmm.clip_grad_norm(torch.nn.Parameter(z), 1.0, 3.0)):
        with pytest.raises(ValueError):
            bad()
    p = torch.nn.Parameter(z)
    p.grad = torch.ones_like(z)
    with pytest.raises(ValueError, match="GPU"):
        lpmm.clip_grad_norm([p], 1.0)


@pytest.mark.parametrize("default", [torch.float64, torch.bfloat16])
def test_numbers_under_another_default_type(default):
    """sample() draws its own in float32, whatever torch's default type is: what is refused is that these logits are not on a GPU"""
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        with pytest.raises(ValueError, match="GPU"):
            lpmm.sample(torch.zeros(2, 10, dtype=torch.float32))
    finally:
        torch.set_default_dtype(before)


def test_clipping_without_a_norm():
    """None is not a norm to be allocated, whose value would be whatever was there"""
    plan = lpmm.GradPlan([], [], torch.zeros(256, dtype=torch.uint8), B.GradPlanHost(256, 0, 0, 12, 1))
    with pytest.raises(ValueError, match="norm"):
        lpmm.lpmm_grad_clip(plan, None, 1.0)
    for bad in (torch.zeros(2), torch.zeros(1, dtype=torch.float64), torch.zeros(())):
        with pytest.raises(ValueError, match="norm"):
            lpmm.lpmm_grad_clip(plan, bad, 1.0)
