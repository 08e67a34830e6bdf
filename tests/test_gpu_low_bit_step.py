"""A training step of 8-bit products, clipped gradients and the 4-bit optimizer, and tokens drawn from what it trains: each through the modules, and together."""
import math
import weakref

import pytest
import torch

import f8_util as f8
import paper_2309_01507_amd as lpmm
import sample_util
from conftest import progress

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def norm64(grads):
    return float(torch.cat([g.detach().cpu().double().reshape(-1) for g in grads]).square().sum().sqrt())


def parameters(dtype=torch.float32):
    g = torch.Generator(device=DEV).manual_seed(1)
    out = []
    for shape in ((70, 130), (5000,), (3,), (9, 8, 7)):
        p = torch.nn.Parameter(torch.randn(shape, generator=g, device=DEV))
        p.grad = torch.randn(shape, generator=g, device=DEV)
        out.append(p)
    return out


@pytest.mark.parametrize("norm_type", [2.0, float("inf")])
def test_clip_grad_norm(norm_type):
    """The function and the optimizer's method against 64 bits: a norm rounded to fp32; values by a factor rounded to fp32 from it, and one product"""
    for way in ("function", "method", "method again"):
        ps = parameters()
        ps.append(torch.nn.Parameter(torch.zeros(4, device=DEV)))
        before = [p.grad.clone() for p in ps[:-1]]
        opt = lpmm.SGDM4bit(ps[:-1], lr=0.1)
        want = norm64(before) if norm_type == 2.0 else max(float(g.abs().max()) for g in before)
        if way == "function":
            norm = lpmm.clip_grad_norm(ps, 0.5, norm_type)
        else:
            if way == "method again":
                opt.clip_grad_norm(100 * want, norm_type)
                assert all(torch.equal(p.grad, b) for p, b in zip(ps, before))
            norm = opt.clip_grad_norm(0.5, norm_type)
        assert abs(float(norm) - want) <= 2.0 ** -23 * want
        for p, b in zip(ps, before):
            scaled = b.cpu().double() * (0.5 / (want + 1e-6))
            assert bool(((p.grad.cpu().double() - scaled).abs() <= 4 * 2.0 ** -24 * scaled.abs()).all()), way
    one = parameters()[0]
    assert abs(float(lpmm.clip_grad_norm(one, 1e9)) - norm64([one.grad])) <= 2.0 ** -23 * norm64([one.grad])
    assert float(lpmm.clip_grad_norm([torch.nn.Parameter(torch.zeros(3, device=DEV))], 1.0)) == 0.0


@pytest.mark.parametrize("capturable", [False, True])
def test_a_step_that_clips(capturable):
    """max_norm is a clip in front of the step: the same bits as the two calls; and none that limits nothing"""
    mine, theirs, plain = parameters(), parameters(), parameters()
    a = lpmm.AdamW4bit(mine, lr=1e-2, max_norm=0.7, capturable=capturable)
    b = lpmm.AdamW4bit(theirs, lr=1e-2, capturable=capturable)
    c = lpmm.AdamW4bit(plain, lr=1e-2, max_norm=1e9, capturable=capturable)
    d_params = parameters()
    d = lpmm.AdamW4bit(d_params, lr=1e-2, capturable=capturable)
    for step in range(3):
        for ps in (mine, theirs, plain, d_params):
            g = torch.Generator(device=DEV).manual_seed(step)
            for p in ps:
                p.grad.copy_(torch.randn(p.shape, generator=g, device=DEV))
        b.clip_grad_norm(0.7)
        for o in (a, b, c, d):
            o.step()
        for p, q, r, s in zip(mine, theirs, plain, d_params):
            assert torch.equal(p, q) and torch.equal(r, s) and torch.equal(p.grad, q.grad)


def test_a_captured_step_that_clips():
    """Replays with other gradients in the same place, against eager steps"""
    mine, theirs = parameters(), parameters()
    a = lpmm.AdamW4bit(mine, lr=1e-2, max_norm=0.3, capturable=True)
    b = lpmm.AdamW4bit(theirs, lr=1e-2, max_norm=0.3, capturable=True)
    a.step(), b.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for step in range(4):
        g = torch.Generator(device=DEV).manual_seed(step)
        for p, q in zip(mine, theirs):
            p.grad.copy_((0.1 + step) * torch.randn(p.shape, generator=g, device=DEV))
            q.grad.copy_(p.grad)
        graph.replay()
        b.step()
        assert all(torch.equal(p, q) for p, q in zip(mine, theirs))
        torch.randn(1000, device=DEV).sum().item()


def test_gradients_that_move():
    """zero_grad(set_to_none=True) gives new gradients each time: the list follows"""
    ps = parameters()
    opt = lpmm.AdamW4bit(ps, lr=1e-3, max_norm=0.5)
    for step in range(3):
        for p in ps:
            p.grad = torch.randn(p.shape, device=DEV) + step
        opt.step()
        assert abs(norm64([p.grad for p in ps]) - 0.5) < 1e-5
        opt.zero_grad(set_to_none=True)


def test_sample_of_any_shape():
    g = torch.Generator(device=DEV).manual_seed(4)
    z = torch.randn(2, 3, 500, generator=g, device=DEV)
    u = torch.rand(2, 3, generator=g, device=DEV)
    heat = torch.rand(2, 3, generator=g, device=DEV) + 0.5
    k = torch.randint(0, 9, (2, 3), generator=g, device=DEV, dtype=torch.int32)
    tokens, logprob = lpmm.sample(z, heat, k, 0.9, 0.01, u=u)
    assert tokens.shape == logprob.shape == (2, 3)
    flat = lambda x: x.reshape(6, *x.shape[2:]).cpu()
    sample_util.check(flat(z), flat(u), flat(heat), flat(k), 0.9, 0.01, flat(tokens), flat(logprob), "(2, 3)")
    t = z.permute(1, 0, 2)                                   # not contiguous
    turned, _ = lpmm.sample(t, heat.t(), k.t(), 0.9, 0.01, u=u.t())
    assert torch.equal(turned, tokens.t())
    again = [lpmm.sample(z, generator=torch.Generator(device=DEV).manual_seed(7))[0] for _ in range(2)]
    assert torch.equal(*again)
    one, lp = lpmm.sample(z[0, 0], temperature=0.0)
    assert one.shape == () and int(one) == int(z[0, 0].argmax()) and float(lp) == 0.0
    with pytest.raises(ValueError):
        lpmm.sample(z, u=u[0])
    with pytest.raises(ValueError):
        lpmm.sample(z, heat[0], u=u)


def test_draws_follow_the_distribution():
    """20000 draws of one distribution: counts within 5 standard deviations of what the kept probabilities say, nothing else drawn"""
    z = torch.tensor([2.0, 1.5, 0.3, -1.0, -4.0, float("-inf")], device=DEV).expand(20000, 6).contiguous()
    tokens, logprob = lpmm.sample(z, 0.8, 4, 0.97, generator=torch.Generator(device=DEV).manual_seed(1))
    w = torch.exp(z[0, :4].cpu().double() / 0.8)
    order = torch.cumsum(w, 0) - w
    w[order >= 0.97 * w.sum()] = 0
    p = w / w.sum()
    count = torch.bincount(tokens.cpu(), minlength=6).double()
    assert bool((count[4:] == 0).all())
    assert bool(((count[:4] - 20000 * p).abs() <= 5 * (20000 * p * (1 - p)).sqrt()).all())
    assert bool((logprob.cpu().double() - p.log()[tokens.cpu()]).abs().max() < 1e-6)


def test_together():
    """A layer of 8-bit products is trained on the distillation loss with clipped gradients by 4-bit AdamW, and writes tokens by drawing: its gradient is the
    formula's, the norm is that of the gradient, and every token could be drawn."""
    g = torch.Generator(device=DEV).manual_seed(2)
    tokens, width, vocab = 160, 256, 1500
    teacher = torch.randn(vocab, width, generator=g, device=DEV) / 16
    layer = lpmm.F8Linear.from_weight(teacher + 0.02 * torch.randn(vocab, width, generator=g, device=DEV))
    opt = lpmm.AdamW4bit(layer.parameters(), lr=1e-3, max_norm=0.05)
    for step in range(3):
        progress(f"step {step}")
        x = torch.randn(tokens, width, generator=g, device=DEV).bfloat16()
        top, index = torch.topk(x.float() @ teacher.t(), 20, dim=1)
        opt.zero_grad()
        z = layer(x)
        z.retain_grad()
        lpmm.distill_loss(z, top, index, 2.0).sum().backward()
        f8.check_product(layer.weight.grad, f8.quantize(z.grad.cpu().t(), 1)[0], f8.quantize(x.cpu().t(), 1)[0], "dW")
        before, weight = norm64([layer.weight.grad]), layer.weight.detach().clone()
        assert before > 0.05
        opt.step()
        assert abs(norm64([layer.weight.grad]) - 0.05 * before / (before + 1e-6)) < 1e-6
        assert not torch.equal(weight, layer.weight)
    with torch.no_grad():
        packed = lpmm.lpmm_f8_quant(layer.weight.detach(), 128)
        x = torch.randn(9, width, generator=g, device=DEV).bfloat16()
        z = lpmm.lpmm_f8_linear(x, packed)
        f8.check_product(z, f8.quantize(x.cpu(), 1)[0], f8.unpack(packed)[0], "logits")
        u = torch.rand(9, generator=g, device=DEV)
        drawn, logprob = lpmm.sample(z, 0.7, 50, 0.9, u=u)
    sample_util.check(z.cpu(), u.cpu(), 0.7, 50, 0.9, 0.0, drawn, logprob, "drawn")


@pytest.mark.parametrize("kind", ["w4", "f8"])
def test_recovery_with_clipping_and_drawing(kind):
    """The command's options run: finite numbers, not how far anything falls"""
    from paper_2309_01507_amd import w4_recovery
    before, after, off = w4_recovery.recover(3, student_kind=kind, max_norm=0.1, temperature=0.9, top_p=0.95)
    assert all(math.isfinite(v) for v in (before, after, off))


@pytest.mark.parametrize("how", ["max_norm", "method"])
def test_gradients_are_let_go(how):
    """After a clipped step, zero_grad(set_to_none=True) frees the gradients; the next ones may get the same addresses; and autograd knows of what the optimizer's clip wrote"""
    ps = parameters()
    opt = lpmm.AdamW4bit(ps, lr=1e-3, max_norm=0.5 if how == "max_norm" else None)
    for step in range(3):
        for p in ps:
            p.grad = torch.randn(p.shape, device=DEV) + step
        if how == "method":
            opt.clip_grad_norm(0.5)
        opt.step()
        assert abs(norm64([p.grad for p in ps]) - 0.5) < 1e-5
        old, size = [weakref.ref(p.grad) for p in ps], sum(p.grad.numel() * 4 for p in ps)
        before = torch.cuda.memory_allocated()
        opt.zero_grad(set_to_none=True)
        assert all(r() is None for r in old) and torch.cuda.memory_allocated() <= before - size
    x = torch.randn(ps[0].shape, device=DEV, requires_grad=True)
    for p in ps:
        p.grad = torch.randn(p.shape, device=DEV)
    for again in range(2):
        y = (x * ps[0].grad).sum()
        opt.clip_grad_norm(0.1)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float64])
@pytest.mark.parametrize("make", [lambda ps: lpmm.AdamW4bit(ps, lr=1e-2), lambda ps: lpmm.AdamW4bit(ps, lr=1e-2, capturable=True), lambda ps: lpmm.SGDM4bit(ps, lr=1e-2)])
def test_optimizers_under_another_default_type(make, default):
    """States and rates that kernels take as float32 are that whatever torch's default type is: the same bits"""
    mine, theirs = parameters(), parameters()
    b = make(theirs)
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        a = make(mine)
        for _ in range(2):
            a.step()
    finally:
        torch.set_default_dtype(before)
    for _ in range(2):
        b.step()
    assert all(torch.equal(p, q) for p, q in zip(mine, theirs))
    floats = [x for st in a.state_buffers() for x in a._tensors_of(st).values() if x.is_floating_point()]
    assert floats and all(x.dtype == torch.float32 for x in floats)
