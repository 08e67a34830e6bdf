"""4-bit weights on the GPU where a kernel's way of holding its operands shows: single products, infinite weights and gradients."""
import pytest
import torch

import paper_2309_01507_amd as lpmm
import w4_util as ref
from conftest import progress
from w4_util import DEV

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
INF = float("inf")


def weights(rows, cols, group, seed):
    q, packed, scales = ref.random_weights(rows, cols, group, seed)
    return lpmm.WeightsW4(rows, cols, group, packed.to(DEV), scales.to(DEV)), ref.VALUES[q], scales


def strided(x, extra, offset=0):
    """The same matrix on the GPU with `extra` elements of NaN between its rows, `offset` elements off an aligned start"""
    t, n = x.shape
    buf = torch.full((t * (n + extra) + offset,), float("nan"), dtype=x.dtype, device=DEV)
    view = buf[offset:].view(t, n + extra)[:, :n]
    view.copy_(x)
    return view


# On both routes (rows on 16-byte boundaries or not) tiles of 64, 128 and 256 tokens, with and without splits of the reduction
@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("t,rows,cols,group", [(5, 64, 200, 32), (100, 96, 130, 64), (300, 160, 256, 128), (1100, 96, 2050, 32), (8100, 160, 2040, 64)])
def test_gradient_of_the_input_does_not_round_the_weights(t, rows, cols, group, offset):
    """One element of dy a token, so that an element of dx is one product.  Of value * scale 2^-13 may be lost, and 2^-20 be added, on
    the way; what remains is the rounding of the result."""
    progress(f"w4 dx single products {t} x {rows} x {cols} group {group} offset {offset}")
    w, values, scales = weights(rows, cols, group, 3)
    full = values * ref.spread(scales, group, cols)
    g = torch.Generator().manual_seed(4)
    at, size = torch.arange(t) % rows, torch.randn(t, generator=g).to(BF16)
    dy = torch.zeros(t, rows, dtype=BF16)
    dy[torch.arange(t), at] = size
    want = size.double()[:, None] * full[at]
    tol = ref.bound(BF16, want, want.abs(), 4, 2.0 ** -13 + 2.0 ** -20)
    ref.assert_within(lpmm.lpmm_w4_linear_dx(strided(dy, 8, offset), w), want, tol, "dx")


def check_what_is_not_finite(t, dtype, offset):
    """Infinite and NaN scales, and such elements of dy, reach the elements of dx that the formula lets them reach, with its sign."""
    rows, cols, group = 96, 200, 32
    w, values, scales = weights(rows, cols, group, 6)
    scales = scales.abs() + 0.01
    scales[5, 0], scales[40, 3], scales[41, 2], scales[90, 6], scales[17, 1] = INF, -INF, 5.5e37, INF, float("nan")
    w = lpmm.WeightsW4(rows, cols, group, w.codes, scales.to(DEV))
    full = values * ref.spread(scales, group, cols)
    g = torch.Generator().manual_seed(2)
    dy = torch.randn(t, rows, generator=g)
    dy[torch.rand(t, rows, generator=g) < 0.2] = 1.0           # nothing left in lower terms
    dy[:, 41] = 0.5                                            # no sum of what is finite overflows
    dy = dy.to(dtype)
    dy[0, 3], dy[1, 95], dy[2, 40], dy[3, 7] = INF, -INF, INF, float("nan")
    got, want = lpmm.lpmm_w4_linear_dx(strided(dy, 8, offset), w).cpu(), dy.double() @ full
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf].double(), want[inf])


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("t", [4, 150, 300])
def test_infinite_weights_and_gradients_bf16(t, offset):
    check_what_is_not_finite(t, BF16, offset)


@pytest.mark.parametrize("t", [4, 65, 300])
def test_infinite_weights_and_gradients_fp32(t):
    check_what_is_not_finite(t, F32, 0)


# Each kind of tile: few tokens, runs split or shared among waves, large tiles; on 16-byte boundaries and off them
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("t,rows", [(3, 70), (20, 70), (40, 9000), (64, 9000), (300, 9000)])
def test_infinite_scales_in_the_product(t, rows, group, dtype):
    """A group's sum times its scale: an infinite scale, that of a short last group among them, gives infinity with the sum's sign."""
    cols = 200
    progress(f"w4 infinite scales {t} x {rows} x {cols} group {group} {dtype}")
    w, values, scales = weights(rows, cols, group, 8)
    last = scales.shape[1] - 1
    scales[3, last], scales[66, last], scales[5, 0], scales[9, 1] = INF, -INF, INF, float("nan")
    w = lpmm.WeightsW4(rows, cols, group, w.codes, scales.to(DEV))
    g = torch.Generator().manual_seed(5)
    x = torch.randn(t, cols, generator=g).to(dtype)
    want = sum(scales[:, j].double()[None, :] * (x[:, j * group:(j + 1) * group].double() @ values[:, j * group:(j + 1) * group].t())
               for j in range(last + 1))
    for offset in (0, 1):
        got = lpmm.lpmm_w4_linear(strided(x, 8, offset), w).cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        inf = torch.isinf(want)
        assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf].double(), want[inf])
