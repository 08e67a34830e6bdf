"""The products' and gradients' kernels over the ranges that each of them is taken for: rows of 9 to 40 runs of 128 for few tokens, several tiles of
rows a workgroup, rows that end within a run in tiles of every size, many steps of the largest tiles.  Against 64-bit products."""
import pytest
import torch

import paper_2309_01507_amd as lpmm
import w4_util as ref
from conftest import progress
from w4_util import DEV

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
GROUPS = (32, 64, 128)


def weights(rows, cols, group, seed):
    """(weights, values * scales in 64 bits), made on the GPU: all 16 codes, scales of both signs, some 0"""
    g = torch.Generator(device=DEV).manual_seed(seed)
    q = torch.randint(0, 16, (rows, cols), generator=g, device=DEV, dtype=torch.uint8)
    byte, shift = ref.place(torch.arange(-(-cols // 128) * 128))
    packed = torch.zeros(rows, -(-cols // 128) * 64, dtype=torch.uint8, device=DEV)
    for want in (0, 4):
        at = torch.nonzero(shift[:cols] == want).flatten()
        packed[:, byte[at].to(DEV)] |= q[:, at.to(DEV)] << want
    scales = 0.02 * torch.randn(rows, -(-cols // group), generator=g, device=DEV).exp()
    scales *= torch.where(torch.rand(scales.shape, generator=g, device=DEV) < 0.1, -1.0, 1.0)
    scales[torch.rand(scales.shape, generator=g, device=DEV) < 0.05] = 0.0
    full = ref.VALUES.to(DEV)[q.int()] * ref.spread(scales, group, cols)
    return lpmm.WeightsW4(rows, cols, group, packed.view(-1), scales), full


def rows_apart(t, cols, dtype, extra, offset, seed):
    """Random rows with `extra` elements of NaN between them, `offset` elements off an aligned start"""
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(t, cols, generator=g, device=DEV) * torch.exp(0.5 * torch.randn(1, cols, generator=g, device=DEV))
    buf = torch.full((t * (cols + extra) + offset,), float("nan"), dtype=dtype, device=DEV)
    view = buf[offset:].view(t, cols + extra)[:, :cols]
    view.copy_(x)
    return view


def compare(got, a, b, steps, operand, what):
    want, mag = a @ b, a.abs() @ b.abs()
    ref.assert_within(got, want.cpu(), ref.bound(got.dtype, want, mag, steps, operand).cpu(), what)


def check_linear(t, rows, cols, group, dtype, extra, offset):
    progress(f"w4 ranges {t} x {rows} x {cols} group {group} {dtype} offset {offset}")
    w, full = weights(rows, cols, group, rows + cols)
    x = rows_apart(t, cols, dtype, extra, offset, t)
    compare(lpmm.lpmm_w4_linear(x, w), x.double(), full.t().contiguous(), cols + 4, 0.0, "y")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("cols", [1160, 2048, 2056, 4096, 4100, 5000])
@pytest.mark.parametrize("t", [1, 7, 16, 32])
def test_few_tokens_by_rows_of_every_length(t, cols, group, dtype):
    check_linear(t, 40, cols, group, dtype, 0, 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("t,rows,cols", [(1, 9001, 640), (16, 9001, 1000), (7, 9001, 2048), (16, 9001, 2056), (7, 9001, 5000), (3, 17000, 2056),
                                         (7, 17000, 4100), (1, 20000, 9000)])
def test_few_tokens_by_many_rows(t, rows, cols, group, dtype):
    """Workgroups that take several tiles of rows, with x in registers from tile to tile or read again for each of several chunks"""
    check_linear(t, rows, cols, group, dtype, 0, 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("t,rows,cols", [(20, 8100, 1000), (32, 8100, 2056), (17, 8100, 4100)])
def test_up_to_32_tokens_off_alignment(t, rows, cols, group, dtype):
    check_linear(t, rows, cols, group, dtype, 3, 1)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("t,rows,cols", [(20, 300, 1000), (33, 4500, 648), (64, 9000, 392), (64, 9000, 1160), (300, 700, 1400), (700, 6000, 136), (700, 6000, 584),
                                         (1030, 5000, 968)])
def test_rows_that_end_within_a_run(t, rows, cols, group, dtype, offset):
    check_linear(t, rows, cols, group, dtype, 8, offset)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("t,rows,cols,group", [(8100, 160, 2040, 32), (8100, 224, 2040, 128), (2100, 96, 2000, 64), (2100, 160, 2000, 32), (1030, 4128, 136, 64),
                                               (150, 2080, 1000, 128), (16, 3000, 700, 32)])
def test_gradient_of_the_input_in_many_steps(t, rows, cols, group, dtype, offset):
    progress(f"w4 ranges dx {t} x {rows} x {cols} group {group} {dtype} offset {offset}")
    w, full = weights(rows, cols, group, rows + cols)
    dy = rows_apart(t, rows, dtype, 8 + -rows % 8, offset, t)
    # bf16: value * scale is held to 2^-13, and 2^-20 too large
    compare(lpmm.lpmm_w4_linear_dx(dy, w), dy.double(), full, rows + 4, 2.0 ** -13 + 2.0 ** -20 if dtype == BF16 else 0.0, "dx")
