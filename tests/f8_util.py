"""Plain 64-bit forms of the 8-bit matrices' operators, on the CPU, written from the format and the formulas in include/lpmm4.h."""
import math

import torch

DEV = "cuda:0"


def scale_of(part):
    """The byte of a block (CPU, 64 bits)"""
    fine = part[torch.isfinite(part)]
    top = float(fine.abs().max()) if fine.numel() else 0.0
    if top == 0.0:
        return 0
    e = math.frexp(top / 448)[1] - 1                                      # 2^e <= top / 448 < 2^(e + 1)
    while top > 448 * 2.0 ** e:
        e += 1
    while top <= 448 * 2.0 ** (e - 1):
        e -= 1
    return max(-127, e) + 127


def quantize(x, tile):
    """x: CPU matrix of any float type -> (values in 64 bits, NaN where there is no code; scale bytes [blocks of rows, blocks of columns])"""
    x = x.double()
    rows, cols = x.shape
    scales = torch.zeros(-(-rows // tile), -(-cols // 128), dtype=torch.long)
    power = torch.zeros_like(x)
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            r, c = slice(i * tile, (i + 1) * tile), slice(j * 128, (j + 1) * 128)
            scales[i, j] = scale_of(x[r, c])
            power[r, c] = 2.0 ** (int(scales[i, j]) - 127)
    a = x / power                                                         # exact: a power of two
    step = 2.0 ** (torch.floor(torch.log2(a.abs().clamp(min=2.0 ** -6))) - 3)
    # torch.log2 is exact at powers of two and monotone between, in 64 bits
    value = torch.round(a / step) * step * power
    value[~torch.isfinite(x)] = math.nan
    return value, scales


def unpack(m):
    """Values in 64 bits of what a kernel wrote, the codes read bit by bit; the padding is checked"""
    codes, scales = m.codes.cpu().long(), m.scales.cpu().long()
    assert codes.shape == (m.rows, -(-m.cols // 128) * 128)
    assert bool((codes[:, m.cols:] == 0).all()), "the rest of a row is 0"
    blocks = -(-m.cols // 128)
    if m.tile == 1:
        assert scales.shape == (blocks, -(-m.rows // 4) * 4)
        assert bool((scales[:, m.rows:] == 0).all()), "the rest of a row of scales is 0"
        scales = scales[:, :m.rows].t()
    else:
        assert scales.shape == (-(-m.rows // 128), -(-blocks // 4) * 4)
        assert bool((scales[:, blocks:] == 0).all()), "the rest of a row of scales is 0"
    power, part = codes >> 3 & 15, (codes & 7).double()
    v = torch.where(power > 0, (8 + part) * 2.0 ** (power.double() - 10), part * 2.0 ** -9)
    v[(codes & 127) == 127] = math.nan
    v = torch.where(codes > 127, -v, v)
    rows = torch.arange(m.rows) // m.tile
    scale = scales[rows][:, torch.arange(m.cols) // 128]
    return v[:, :m.cols] * 2.0 ** (scale.double() - 127), scales[:, :blocks]


def same(got, want):
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


def bound(dtype, want, magnitude, steps):
    """How far a product may be off: its rounding (half a unit: 2^-8 in bf16, 2^-24 in fp32), and `steps` roundings of fp32 sums whose terms' magnitudes
    add up to `magnitude`.  In bf16 also what the matrix instructions on 8 bits cut off: each of the eight products that are added up at once ends
    2^-13 below the largest of them (256 and 127 times 2^-6 give 257.875: seven are lost), so at most 8 * 2^-13 of that one, which is among the magnitudes."""
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    return u * want.abs() + (1 + u) * magnitude * (steps * 2.0 ** -24 + (2.0 ** -10 if dtype == torch.bfloat16 else 0.0)) + 1e-37


def assert_within(got, want, tol, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, f"{what}: shape {tuple(got.shape)}"
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine].nan_to_num(0.0), want[~fine].nan_to_num(0.0)), f"{what}: infinities"
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, \
        f"{what}: {int((over > 0).sum())} of {over.numel()} too far off, worst by {float(over.max()):.3g}"


def check_product(got, a, b, what):
    """a b^T of values in 64 bits against what a kernel gave.  fp32 sums of n terms in any order take at most n roundings; and, sharper for
    results of 16 bits, the error as a whole: each is rounded by at most 2^-8 of itself."""
    want, magnitude = a @ b.t().contiguous(), a.abs().nan_to_num(0.0) @ b.abs().nan_to_num(0.0).t().contiguous()
    assert_within(got, want, bound(got.dtype, want, magnitude, a.shape[1]), what)
    fine = torch.isfinite(want)
    off, size = (got.detach().cpu().double() - want)[fine], want[fine]
    if got.dtype == torch.bfloat16 and off.numel() >= 100 and a.shape[1] >= 32:
        assert float(off.norm()) <= (2.0 ** -8 + 2.0 ** -12) * float(size.norm()), what
