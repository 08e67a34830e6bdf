"""Plain 64-bit forms of the 4-bit weights' operators and of distillation, on the CPU, written from the formulas in
include/lpmm4.h."""
import math

import torch

VALUES = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)
MIDPOINTS = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)
DEV = "cuda:0"


def place(k):
    """(byte of its row, shift) of element k's code"""
    d = k % 128 // 8
    return k // 128 * 64 + ((d % 4) * 4 + d // 4) * 4 + k % 8 // 2, k % 2 * 4


def unpack(codes, rows, cols):
    c = codes.cpu().view(rows, -1).long()
    k = torch.arange(cols)
    byte, shift = place(k)
    return (c[:, byte] >> shift) & 15


def pack(q):
    """codes (one each) -> rows of bytes with padding"""
    rows, cols = q.shape
    out = torch.zeros(rows, -(-cols // 128) * 64, dtype=torch.long)
    k = torch.arange(cols)
    byte, shift = place(k)
    out.index_add_(1, byte, q.long() << shift)          # two codes of a byte do not overlap
    return out.to(torch.uint8).reshape(-1)


def quantize(w, group):
    """w: CPU tensor of any float type -> (codes one each, fp32 scales); every comparison is exact in 64 bits"""
    rows, cols = w.shape
    w = w.double()
    groups = -(-cols // group)
    scales = torch.zeros(rows, groups)
    q = torch.zeros(rows, cols, dtype=torch.long)
    for j in range(groups):
        part = w[:, j * group:(j + 1) * group]
        top = part.abs().amax(dim=1).float()
        s = torch.where(top < 2.0 ** -100, torch.zeros_like(top), (top.double() / 6).float())
        bad = ~torch.isfinite(part).all(dim=1)
        s[bad] = math.nan
        scales[:, j] = s
        count = sum((part.abs() > m * s.double()[:, None]).long() for m in MIDPOINTS)
        count[(s == 0) | bad] = 0
        q[:, j * group:(j + 1) * group] = count + 8 * ((part < 0) & (count > 0)).long()
    return q, scales


def spread(scales, group, cols):
    return scales.double().repeat_interleave(group, dim=1)[:, :cols]


def group_sums(m, group):
    rows, cols = m.shape
    return torch.nn.functional.pad(m, (0, -(-cols // group) * group - cols)).view(rows, -1, group).sum(dim=2)


def random_weights(rows, cols, group, seed):
    """(codes one each, packed bytes, scales): all 16 codes, scales of different size and sign, some 0"""
    g = torch.Generator().manual_seed(seed)
    q = torch.randint(0, 16, (rows, cols), generator=g)
    scales = 0.02 * torch.randn(rows, -(-cols // group), generator=g).exp()
    scales *= torch.where(torch.rand(scales.shape, generator=g) < 0.1, -1.0, 1.0)
    scales[torch.rand(scales.shape, generator=g) < 0.05] = 0.0
    return q, pack(q), scales


def bound(out_dtype, want, magnitude, steps, operand=0.0):
    """How far a kernel may be from `want`: one rounding to its type, `steps` roundings of fp32 sums whose terms have magnitudes that
    add up to `magnitude`, and a relative rounding of the operands.  Half a unit in the last place is 2^-8 in bf16 and 2^-24 in fp32."""
    u = 2.0 ** -8 if out_dtype == torch.bfloat16 else 2.0 ** -24
    return u * want.abs() + (1 + u) * magnitude * (steps * 2.0 ** -24 + operand) + 1e-37


def assert_within(got, want, tol, what):
    got = got.cpu().double()
    assert got.shape == want.shape, f"{what}: shape {tuple(got.shape)}"
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), f"{what}: infinities"
    fine = torch.isfinite(want)
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, \
        f"{what}: {int((over > 0).sum())} of {over.numel()} too far off, worst by {float(over.max()):.3g}"


def distill(z, top, index, tau, grad):
    """(loss, lse, dz, the p's) in 64 bits; z, top: CPU"""
    z, top, grad = z.double(), top.double(), grad.double()
    t, v = z.shape
    loss, lse, dz = torch.zeros(t).double(), torch.zeros(t).double(), torch.zeros(t, v).double()
    for r in range(t):
        slots = [(int(i), float(u) / tau) for i, u in zip(index[r], top[r]) if 0 <= int(i) < v]
        if not slots:
            continue
        x = z[r] / tau
        lse[r] = torch.logsumexp(x, 0)
        u = torch.tensor([b for _, b in slots], dtype=torch.float64)
        log_p = torch.log_softmax(u, 0)
        d = torch.exp(x - lse[r])
        total = 0.0
        for (i, _), lp in zip(slots, log_p.tolist()):
            p = math.exp(lp)
            if p != 0:
                total += p * (lp - (float(x[i]) - float(lse[r])))
            d[i] -= p
        loss[r] = tau * tau * total
        dz[r] = grad[r] * tau * d if float(grad[r]) != 0 else 0.0
    return loss, lse, dz
