"""Distillation from a teacher's top logits on the GPU against a plain 64-bit form."""
import ctypes

import pytest
import torch

import paper_2309_01507_amd as lpmm
import w4_util as ref
from conftest import progress
from w4_util import DEV

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
INF = float("inf")


def inputs(t, v, slots, dtype, seed, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    z = (spread * torch.randn(t, v, generator=g)).to(dtype)
    top = 4.0 + 1.5 * torch.randn(t, slots, generator=g)
    index = torch.stack([torch.randperm(v, generator=g)[:slots] if slots <= v else
                         torch.randint(0, v, (slots,), generator=g) for _ in range(t)])
    grad = torch.rand(t, generator=g) / t
    return z, top, index, grad


def check(z, top, index, tau, grad, what, dz_of=None):
    """Both ways of calling, against 64 bits.  z is exact on both sides; the exponent z / tau - lse has an error of a few units of 2^-24
    times its parts, which becomes a relative error of the probability; sums of up to v terms of one sign
    err by a few units of the tree's depth, taken as 64."""
    loss64, lse64, dz64 = ref.distill(z, top, index, tau, grad)
    t, v = z.shape
    x = z.double() / tau
    finite = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x))
    # z / tau: 1.5 units (1 / tau rounded, the product rounded); lse: rounded once, with an error of the sum
    arg = 2.0 ** -24 * (2 * finite + 2 * lse64.abs()[:, None].nan_to_num(0, 0, 0) + 64)
    p64 = torch.exp(x - lse64[:, None])
    u_out = 2.0 ** -8 if z.dtype == BF16 else 2.0 ** -24
    # p_j: the same from the teacher's side
    tp = torch.zeros(t, v).double()
    size = torch.zeros(t).double()
    for r in range(t):
        ok = (index[r] >= 0) & (index[r] < v)
        if bool(ok.any()):
            u = torch.softmax(top[r][ok].double() / tau, 0)
            tp[r].index_add_(0, index[r][ok], u)
            both = finite[r][index[r][ok]] + float(lse64[r].nan_to_num(0, 0, 0).abs())
            term = u * (both + 2 * (top[r][ok].double() / tau).abs() + 16)
            size[r] = float(term[u > 0].sum())                        # terms with p = 0 are not computed
    scale = (grad.double() * tau).abs()[:, None]
    top_arg = 2.0 ** -24 * (4 * top.double().abs().amax(dim=1, keepdim=True).nan_to_num(0, 0, 0) / tau + 64)
    tol_dz = u_out * dz64.abs() + scale * (p64 * arg + tp * top_arg).nan_to_num(0, 0, 0) * (1 + u_out) + 1e-37
    tol_loss = tau * tau * (2.0 ** -24 * 8 * size + 2.0 ** -24 * 80) + 2.0 ** -22 * loss64.abs()
    zd, td, xd, gd = z.to(DEV), top.to(DEV), index.to(DEV), grad.to(DEV)
    loss, lse = lpmm.lpmm_distill_loss(zd, td, xd, tau)
    dz = lpmm.lpmm_distill_grad(zd, td, xd, tau, lse, gd)
    both_loss, both_dz = lpmm.lpmm_distill_loss_grad(zd, td, xd, tau, gd)
    torch.cuda.synchronize()
    assert torch.equal(zd.cpu().view(torch.uint8), z.view(torch.uint8)), "the logits were changed"
    ref.assert_within(lse, lse64, 2.0 ** -24 * (2 * lse64.abs() + 2 * finite.amax(dim=1) + 64), what + " lse")
    for name, got_loss, got_dz in (("two calls", loss, dz), ("one call", both_loss, both_dz)):
        ref.assert_within(got_loss, loss64, tol_loss, f"{what} {name}: loss")
        ref.assert_within(got_dz, dz64, tol_dz, f"{what} {name}: dz")
    return dz64


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,v,slots,tau", [(1, 1, 1, 1.0), (1, 2, 3, 1.0), (3, 5, 5, 2.0), (2, 63, 8, 1.0), (5, 1000, 1, 0.5),
                                           (4, 4096, 64, 1.0), (7, 8191, 65, 4.0), (3, 8193, 20, 2.0), (2, 32000, 256, 1.0),
                                           (300, 1031, 10, 1.0), (270, 50257, 5, 1.5), (1, 131072, 1024, 1.0), (2, 131073, 64, 1.0),
                                           (260, 70001, 33, 1.0), (1, 300007, 100, 1.0), (600, 40, 7, 3.0)])
def test_against_64_bits(t, v, slots, tau, dtype):
    progress(f"distill {t} x {v}, {slots} slots, tau {tau} {dtype}")
    check(*inputs(t, v, slots, dtype, t + v + slots)[:3], tau, inputs(t, v, slots, dtype, t + v + slots)[3], f"{t} x {v}")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t", [9, 300])
def test_masks_and_padding(t, dtype):
    """Slots that do not count, rows without a teacher (full of NaN and infinities), rows without a gradient, places named twice,
    logits of -infinity and of the type's lowest value, a teacher's -infinity."""
    v, slots = 4099, 12
    z, top, index, grad = inputs(t, v, slots, dtype, 8)
    z[:, v - 100:] = -INF
    index[index >= v - 100] = 7
    z[0, 10:4000] = torch.finfo(dtype).min
    index[1, 4:] = -1
    index[2, ::2] = v                                   # out of range at the upper end
    index[2, 1] = 1 << 40
    index[3] = -1
    z[3] = float("nan")
    index[4] = -5
    z[4, ::3] = INF
    index[5] = 77                                       # one place, twelve times
    index[6, 3:9] = index[6, 2]
    top[6, 5] = -INF
    grad[7] = 0.0
    z[8, 50] = -INF
    index[8] = torch.arange(50, 50 + slots)
    top[8, 0] = -INF                                    # -infinity on both sides: the term is 0
    check(z, top, index, 1.0, grad, "masks")
    # a row whose gradient is 0 has dz 0 whatever its logits hold
    z[7, 5] = float("nan")
    zd, td, xd, gd = z.to(DEV), top.to(DEV), index.to(DEV), grad.to(DEV)
    lse = lpmm.lpmm_distill_loss(zd, td, xd, 1.0)[1]
    for dz in (lpmm.lpmm_distill_grad(zd, td, xd, 1.0, lse, gd), lpmm.lpmm_distill_loss_grad(zd, td, xd, 1.0, gd)[1]):
        assert bool((dz[7] == 0).all()) and bool((dz[3] == 0).all()) and bool((dz[4] == 0).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_what_is_not_finite_shows(dtype):
    """NaN in a logit makes its own row NaN; a teacher's place with a logit of -infinity costs infinitely much."""
    z, top, index, grad = inputs(6, 3000, 8, dtype, 3)
    z[1, 2999] = float("nan")
    z[4, int(index[4, 2])] = -INF
    zd, td, xd, gd = z.to(DEV), top.to(DEV), index.to(DEV), grad.to(DEV)
    loss, lse = lpmm.lpmm_distill_loss(zd, td, xd, 1.0)
    dz = lpmm.lpmm_distill_grad(zd, td, xd, 1.0, lse, gd)
    loss2, dz2 = lpmm.lpmm_distill_loss_grad(zd, td, xd, 1.0, gd)
    for lo, d in ((loss.cpu(), dz.cpu()), (loss2.cpu(), dz2.cpu())):
        assert torch.isnan(lo).tolist() == [False, True, False, False, False, False]
        assert float(lo[4]) == INF
        assert bool(torch.isnan(d[1]).all()) and bool(torch.isfinite(d[[0, 2, 3, 4, 5]]).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,v", [(3, 5000), (280, 2049), (2, 200000)])
def test_in_place_and_rows_apart(t, v, dtype):
    z, top, index, grad = inputs(t, v, 9, dtype, 5)
    index[:, 4] = index[:, 2]
    td, xd, gd = top.to(DEV), index.to(DEV), grad.to(DEV)
    loss, lse = lpmm.lpmm_distill_loss(z.to(DEV), td, xd, 2.0)
    want = lpmm.lpmm_distill_grad(z.to(DEV), td, xd, 2.0, lse, gd)
    want_loss, want_one = lpmm.lpmm_distill_loss_grad(z.to(DEV), td, xd, 2.0, gd)
    def apart():
        buf = torch.full((t, v + 3), float("nan"), dtype=dtype, device=DEV)
        buf[:, :v] = z.to(DEV)
        return buf[:, :v]
    a, b, c = apart(), apart(), apart()
    l2, s2 = lpmm.lpmm_distill_loss(a, td, xd, 2.0)
    assert torch.equal(loss, l2) and torch.equal(lse, s2)
    assert torch.equal(lpmm.lpmm_distill_grad(a, td, xd, 2.0, lse, gd), want)
    assert torch.equal(lpmm.lpmm_distill_grad(a, td, xd, 2.0, lse, gd, a), want)
    l3, d3 = lpmm.lpmm_distill_loss_grad(b, td, xd, 2.0, gd, dz=b)
    assert torch.equal(l3, want_loss) and torch.equal(d3, want_one)
    for buf in (a, b):
        assert bool(torch.isnan(buf.as_strided((t - 1, 3), (v + 3, 1), v)).all())
    out = torch.full((t, v + 8), float("nan"), dtype=dtype, device=DEV)
    lpmm.lpmm_distill_loss_grad(c, td, xd, 2.0, gd, dz=out[:, 1:v + 1])
    assert torch.equal(out[:, 1:v + 1], want_one) and bool(torch.isnan(out[:, v + 1:]).all()) and bool(torch.isnan(out[:, 0]).all())


def test_gradient_against_differences():
    """Central differences of the loss in single logits.  With a step of 1/8 the third derivative (at most 1/4 here, p being a
    probability) leaves an error of at most h^2 / 24 < 7e-4; the loss's rounding, 2^-20, over 2 h adds 4e-6."""
    z, top, index, _ = inputs(40, 200, 6, F32, 11, spread=1.0)
    td, xd = top.to(DEV), index.to(DEV)
    one = torch.ones(40, device=DEV)
    _, dz = lpmm.lpmm_distill_loss_grad(z.to(DEV), td, xd, 1.0, one)
    dz = dz.cpu().double()
    h = 0.125
    g = torch.Generator().manual_seed(1)
    for trial in range(12):
        at = index[:, trial % 6] if trial < 6 else torch.randint(0, 200, (40,), generator=g)
        up, down = z.clone(), z.clone()
        rows = torch.arange(40)
        up[rows, at] += h
        down[rows, at] -= h
        a = lpmm.lpmm_distill_loss(up.to(DEV), td, xd, 1.0)[0].cpu().double()
        b = lpmm.lpmm_distill_loss(down.to(DEV), td, xd, 1.0)[0].cpu().double()
        assert float(((a - b) / (2 * h) - dz[rows, at]).abs().max()) < 1e-3


def test_no_rows():
    z, top = torch.empty(0, 100, device=DEV), torch.empty(0, 4, device=DEV)
    index, grad = torch.empty(0, 4, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    loss, dz = lpmm.lpmm_distill_loss_grad(z, top, index, 1.0, grad)
    assert loss.shape == (0,) and dz.shape == (0, 100)


def test_streams_graphs_and_the_same_bits():
    for t, v in ((3, 60000), (300, 3001)):
        z, top, index, grad = inputs(t, v, 20, BF16, 5)
        zd, td, xd, gd = z.to(DEV), top.to(DEV), index.to(DEV), grad.to(DEV)
        def calls():
            loss, lse = lpmm.lpmm_distill_loss(zd, td, xd, 1.0)
            return (loss, lse, lpmm.lpmm_distill_grad(zd, td, xd, 1.0, lse, gd), *lpmm.lpmm_distill_loss_grad(zd, td, xd, 1.0, gd))
        want = calls()
        assert all(torch.equal(a, b) for a, b in zip(want, calls()))
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            got = calls()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        outs = [torch.zeros_like(a) for a in want]
        ws = torch.empty(max(16, lpmm.lib().lpmm_distill_workspace_bytes(t, v)), dtype=torch.uint8, device=DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lpmm.lpmm_distill_loss(zd, td, xd, 1.0, outs[0], outs[1], ws)
            lpmm.lpmm_distill_grad(zd, td, xd, 1.0, outs[1], gd, outs[2])
            lpmm.lpmm_distill_loss_grad(zd, td, xd, 1.0, gd, outs[3], dz=outs[4], lse=torch.empty(t, device=DEV), workspace=ws)
        for _ in range(4):
            zd.mul_(0.5)
            eager = calls()
            for o in outs:
                o.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, eager))


def test_offsets_beyond_32_bits():
    """Logits of more than 2^32 bytes."""
    t, v = 20000, 131072
    progress("5.2 GB of logits")
    z = torch.zeros(t, v, dtype=BF16, device=DEV)
    rows = [0, 8191, 16384, 16385, t - 1]
    g = torch.Generator().manual_seed(2)
    part = (2.5 * torch.randn(len(rows), v, generator=g)).to(BF16)
    z[rows] = part.to(DEV)
    top, index = torch.randn(t, 8, generator=g), torch.full((t, 8), -1, dtype=torch.int64)
    index[rows] = torch.randint(0, v, (len(rows), 8), generator=g)
    grad = torch.ones(t)
    loss, dz = lpmm.lpmm_distill_loss_grad(z, top.to(DEV), index.to(DEV), 1.0, grad.to(DEV), dz=z)
    loss64, _, dz64 = ref.distill(part, top[rows], index[rows], 1.0, grad[rows])
    assert float((loss.cpu()[rows].double() - loss64).abs().max()) < 1e-4
    ref.assert_within(dz[rows], dz64, 2.0 ** -8 * dz64.abs() + 1e-5 * (dz64.abs() + 1e-4), "dz")
    assert float(loss.cpu().double().sum()) == pytest.approx(float(loss64.sum()), rel=1e-5)


def test_refusals():
    L = lpmm.lib()
    z, top, index, grad = (a.to(DEV) for a in inputs(4, 100, 6, F32, 1))
    out, loss, lse = torch.zeros(4, 100, device=DEV), torch.zeros(4, device=DEV), torch.zeros(4, device=DEV)
    p = lambda t: t.data_ptr()
    args = [p(z), 0, 4, 100, 100, p(top), p(index), 6, 1.0]
    bad = ((0, None), (0, p(z) + 2), (1, 5), (2, -1), (3, 0), (4, 99), (5, None), (6, None), (6, p(index) + 4), (7, 0), (7, 1025), (8, 0.0),
           (8, float("nan")), (8, float("inf")), (8, -1.0), (8, 1e-44))
    for at, value in bad:
        a = list(args)
        a[at] = value
        assert L.lpmm_distill_loss(*a, p(loss), p(lse), None, 0, None) == -1, (at, value)
        assert L.lpmm_distill_grad(*a, p(lse), p(grad), p(out), 100, None) == -1, (at, value)
        assert L.lpmm_distill_loss_grad(*a, p(grad), p(loss), p(lse), p(out), 100, None, 0, None) == -1, (at, value)
    assert L.lpmm_distill_loss(*args, None, p(lse), None, 0, None) == -1
    assert L.lpmm_distill_grad(*args, p(lse), p(grad), p(z), 101, None) == -1       # in place with another stride
    assert L.lpmm_distill_grad(*args, p(lse), None, p(out), 100, None) == -1
    torch.cuda.synchronize()
    for call in (lambda: lpmm.lpmm_distill_loss(z.half(), top, index, 1.0), lambda: lpmm.lpmm_distill_loss(z, top.double(), index, 1.0),
                 lambda: lpmm.lpmm_distill_loss(z, top, index.int(), 1.0), lambda: lpmm.lpmm_distill_loss(z, top[:, :3], index, 1.0),
                 lambda: lpmm.lpmm_distill_loss(z, top.cpu(), index, 1.0), lambda: lpmm.lpmm_distill_loss(z[0], top, index, 1.0),
                 lambda: lpmm.lpmm_distill_loss_grad(z, top, index, 1.0, grad[:2]),
                 lambda: lpmm.lpmm_distill_grad(z, top, index, 1.0, lse, grad, out.bfloat16())):
        with pytest.raises(ValueError):
            call()
