"""Sampling, gradient norms and 8-bit products, as cases that can be measured: which calls, on which sizes, with what inputs,
what a pass cannot do without, and what a correct pass returns.

A case is one of six kinds:
  sample   a token for each row of logits, from a given random number: temperature, the k largest, the share p, at least min_p
  norm     the norm of all gradients of a model, as one vector
  clip     that norm, and the gradients scaled down to a limit, into a flat buffer
  quant    a matrix to 8-bit floating point with a scale for each block of 128, its transpose too, and back to values
  linear   y = x W^T, W in 8 bits, x brought to 8 bits within the call: one token, a few, many
  train    that product with both operands given in full, and its gradients for x and W, each from 8-bit operands

8 bits: E4M3 codes times a power of two, one for each 1 x 128 block ("tile" 1) or 128 x 128 block ("tile" 128): the least that brings the
block's largest element to at most 448.  Rows of codes are padded with zeros to a multiple of 128; the power's exponent + 127 is kept
in a byte, rows of those padded to a multiple of 4 bytes.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
MOST_MACS = 4096 * 11008 * 4096   # of a product
MOST_LOGITS = 2048 * 50257
MOST_GRADS = 360_000_000


def _gated(layers, width, inner, vocab):
    """Gradients of a model with gated feed-forward blocks, "count x elements" for each size"""
    return f"2x{vocab * width} {4 * layers}x{width * width} {3 * layers}x{width * inner} {2 * layers + 1}x{width}"


def _plain_blocks(layers, width, inner, vocab, positions):
    """The same for blocks of two matrices, with biases"""
    return (f"1x{vocab * width} 1x{positions * width} {4 * layers}x{width * width} {2 * layers}x{width * inner} "
            f"{9 * layers + 2}x{width} {layers}x{inner}")


# ---- the cases -------------------------------------------------------------------------------------------------------

def listed():
    return [
        # decoding: one row of logits in full precision; latency counts
        {"name": "sample_t1_v32000_f32", "kind": "sample", "t": 1, "v": 32000, "bf16": False, "temperature": 0.8, "top_k": 0,
         "top_p": 0.95, "min_p": 0.0, "each": False},
        # a serving batch, every request with its own settings, some greedy
        {"name": "sample_t61_v50257_bf16_each", "kind": "sample", "t": 61, "v": 50257, "bf16": True, "temperature": 1.0, "top_k": 50,
         "top_p": 0.9, "min_p": 0.02, "each": True},
        # many rows at once: continuations that a student is then trained on
        {"name": "sample_t2048_v32000_bf16", "kind": "sample", "t": 2048, "v": 32000, "bf16": True, "temperature": 1.0, "top_k": 0,
         "top_p": 0.98, "min_p": 0.0, "each": False},
        # the norm that a training run writes into its log: a 7-billion-parameter model, gradients of 16 bits, over 2^32 elements
        {"name": "norm_7b_bf16", "kind": "norm", "sizes": _gated(32, 4096, 11008, 32000), "bf16": True, "most": False},
        # the scales of a small model in 4 bits: latency counts
        {"name": "clip_scales_f32", "kind": "clip", "sizes": "8x6144 1x30018", "bf16": False, "most": False, "limit": 0.25},
        # a model of 24 layers, a flat gradient buffer of full precision
        {"name": "clip_350m_f32", "kind": "clip", "sizes": _plain_blocks(24, 1024, 4096, 50257, 1024), "bf16": False, "most": False,
         "limit": 1.0},
        # what comes before and after a training step's products: a batch of activations, both ways round
        {"name": "quant_4096x11008_bf16", "kind": "quant", "t": 4096, "k": 11008, "tile": 1, "bf16": True},
        # decoding: one token through a projection
        {"name": "linear_t1_4096x4096_bf16", "kind": "linear", "t": 1, "n": 4096, "k": 4096, "bf16": True},
        # a ragged batch through an odd output head, in full precision
        {"name": "linear_t77_50257x1024_f32", "kind": "linear", "t": 77, "n": 50257, "k": 1024, "bf16": False},
        # a prompt batch through a feed-forward matrix
        {"name": "linear_t4096_11008x4096_bf16", "kind": "linear", "t": 4096, "n": 11008, "k": 4096, "bf16": True},
        # a small model's training step, a ragged number of tokens
        {"name": "train_t333_2304x768_f32", "kind": "train", "t": 333, "n": 2304, "k": 768, "bf16": False},
        # a projection's training step: activations of 16 bits, the weight and its gradient of 32
        {"name": "train_t4096_4096x4096_bf16", "kind": "train", "t": 4096, "n": 4096, "k": 4096, "bf16": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["sample", "sample", "norm", "clip", "quant", "linear", "linear", "train"])
    bf16 = rng.random() < 0.6
    if kind == "sample":
        v = _log_int(rng, 300, 131072)
        t = _log_int(rng, 1, max(1, min(4096, MOST_LOGITS // (v if bf16 else 2 * v))))
        return {"kind": kind, "t": t, "v": v, "bf16": bf16, "temperature": rng.choice([0.6, 0.8, 1.0, 1.3]),
                "top_k": rng.choice([0, 0, _log_int(rng, 1, 300)]), "top_p": rng.choice([1.0, 0.95, 0.9, 0.5]),
                "min_p": rng.choice([0.0, 0.0, 0.05]), "each": rng.random() < 0.4}
    if kind in ("norm", "clip"):
        parts, left = [], _log_int(rng, 2000, MOST_GRADS)
        for _ in range(rng.randint(1, 5)):
            count = _log_int(rng, 1, 60)
            parts.append(f"{count}x{_log_int(rng, 1, max(1, left // count))}")
        case = {"kind": kind, "sizes": " ".join(parts), "bf16": bf16, "most": rng.random() < 0.3}
        if sum(_sizes(case)) > MOST_GRADS:                   # five parts of the largest kind
            case["sizes"] = parts[0]
        if kind == "clip":
            case["limit"] = rng.choice([0.01, 1.0, 1e4])
        return case
    n, k = _log_int(rng, 64, 50257), _log_int(rng, 64, 16384)
    if rng.random() < 0.6:
        k = max(64, k // 64 * 64)
    if rng.random() < 0.5:
        n = max(64, n // 32 * 32)
    if kind == "quant":
        t = min(_log_int(rng, 1, 16384), 4096 * 11008 // k)
        return {"kind": kind, "t": t, "k": k, "tile": rng.choice([1, 128]), "bf16": bf16}
    n = min(n, 32000 * 4096 // k)
    most = max(1, min(8192, MOST_MACS // (n * k * (3 if kind == "train" else 1))))
    if kind == "linear" and rng.random() < 0.4:
        most = min(most, 32)
    return {"kind": kind, "t": _log_int(rng, 1, most), "n": n, "k": k, "bf16": bf16}


def _sizes(case):
    out = []
    for part in case["sizes"].split():
        count, each = part.split("x")
        out += [int(each)] * int(count)
    return out


def _codes_bytes(rows, cols, tile):
    return rows * cols + -(-rows // tile) * -(-cols // 128)


def work(case):
    e = 2 if case["bf16"] else 4
    kind = case["kind"]
    if kind == "sample":
        cells = case["t"] * case["v"]
        # each logit once: a difference, an exponential, a comparison, a sum
        return {"bytes": cells * e + case["t"] * (4 + 8 + 4), "flops": 4 * cells}
    if kind in ("norm", "clip"):
        n = sum(_sizes(case))
        # every element decides the norm, which has to be known before the first is scaled: read twice, written once
        return {"bytes": n * e * (3 if kind == "clip" else 1) + 4, "flops": n * (3 if kind == "clip" else 2)}
    t, k = case["t"], case["k"]
    if kind == "quant":
        return {"bytes": 3 * t * k * e + 2 * (_codes_bytes(t, k, case["tile"]) + _codes_bytes(k, t, case["tile"])), "flops": 8 * t * k}
    n = case["n"]
    if kind == "linear":
        return {"bytes": _codes_bytes(n, k, 128) + e * t * (k + n), "flops": 2 * t * n * k}
    # x, dy read; y, dx written; W read and its gradient written in 32 bits; what is in 8 bits need not leave the chip
    return {"bytes": 2 * e * t * (k + n) + 8 * n * k, "flops": 6 * t * n * k}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    g = _generator(seed)
    dtype = torch.bfloat16 if case["bf16"] else torch.float32
    kind = case["kind"]
    if kind == "sample":
        return _prepare_sample(case, g, dtype)
    if kind in ("norm", "clip"):
        return _prepare_grads(case, g, dtype)
    t, k = case["t"], case["k"]
    if kind == "quant":
        return {"case": case, "x": _activations(t, k, g, dtype)}
    n = case["n"]
    w = torch.randn(n, k, generator=g, device=DEV)
    w *= 0.02 * torch.exp(0.3 * torch.randn(n, 1, generator=g, device=DEV))
    state = {"case": case, "x": _activations(t, k, g, dtype)}
    if kind == "linear":
        codes, scales = _packed(w, 128)
        return state | {"codes": codes, "scales": scales}
    state["x"].requires_grad_()
    dy = torch.randn(t, n, generator=g, device=DEV) * torch.exp(torch.randn(t, 1, generator=g, device=DEV)) * 1e-3
    return state | {"w": w.requires_grad_(), "dy": dy.to(dtype)}


def _activations(t, k, g, dtype):
    x = torch.randn(t, k, generator=g, device=DEV)
    x *= 1.0 + 9.0 * (torch.rand(1, k, generator=g, device=DEV) < 0.005)       # some channels are large
    x[t - t // 50:] = 0.0                                                        # padding tokens
    return x.to(dtype)


def _prepare_sample(case, g, dtype):
    t, v = case["t"], case["v"]
    z = 2.5 * torch.randn(t, v, generator=g, device=DEV)
    z[:, v - v // 50:] = -math.inf                                              # the vocabulary's padding
    state = {"case": case, "z": z.to(dtype), "u": torch.rand(t, generator=g, device=DEV)}
    if case["each"]:
        r = lambda: torch.rand(t, generator=g, device=DEV)
        heat = case["temperature"] * (0.5 + r())
        heat[r() < 0.15] = 0.0                                                  # greedy
        k = 1 + (r() * 2 * max(case["top_k"], 20)).to(torch.int32)
        k[r() < 0.3] = 0                                                        # off
        p = case["top_p"] * (0.8 + 0.2 * r())
        p[r() < 0.3] = 1.0
        least = 0.1 * r()
        least[r() < 0.5] = 0.0
        state |= {"temperature": heat, "top_k": k, "top_p": p, "min_p": least}
    else:
        state |= {key: case[key] for key in ("temperature", "top_k", "top_p", "min_p")}
    return state


def _prepare_grads(case, g, dtype):
    sizes = _sizes(case)
    flat = torch.empty(sum(sizes), dtype=dtype, device=DEV)
    flat.normal_(0.0, 1e-3, generator=g)
    grads, at = [], 0
    for n in sizes:
        grads.append(flat[at:at + n])                     # as buckets hold them: at any boundary
        at += n
    if flat.numel() <= MOST_GRADS:
        for x in grads:                                    # layers differ
            x *= torch.exp(0.5 * torch.randn(1, generator=g, device=DEV))
    out = torch.empty_like(flat) if case["kind"] == "clip" else None
    return {"case": case, "grads": grads, "flat": flat, "out": out,
            "outs": None if out is None else list(out.split(sizes)), "plan": {}}


# ---- one pass --------------------------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2309_01507_amd as lpmm
    c = s["case"]
    kind = c["kind"]
    if kind == "sample":
        return lpmm.lpmm_sample(s["z"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    if kind in ("norm", "clip"):
        if "plan" not in s["plan"]:                        # once, as a training run does
            s["plan"]["plan"] = lpmm.new_grad_plan(s["grads"], s["outs"])
        plan, which = s["plan"]["plan"], lpmm.GRAD_NORM_MAX if c["most"] else lpmm.GRAD_NORM_L2
        if kind == "norm":
            return lpmm.lpmm_grad_norm(plan, which)
        return lpmm.lpmm_grad_norm_clip(plan, c["limit"], which), s["out"]
    if kind == "quant":
        q, qt = lpmm.lpmm_f8_quant_both(s["x"], c["tile"])
        return lpmm.lpmm_f8_dequant(q, s["x"].dtype), lpmm.lpmm_f8_dequant(qt, s["x"].dtype)
    if kind == "linear":
        return lpmm.lpmm_f8_linear(s["x"], lpmm.MatF8(c["n"], c["k"], 128, s["codes"], s["scales"]))
    y = lpmm.f8_linear(s["x"], s["w"])
    return (y.detach(), *torch.autograd.grad(y, (s["x"], s["w"]), s["dy"]))


def _run_plain(s):
    c = s["case"]
    kind = c["kind"]
    if kind == "sample":
        return _plain_sample(s["z"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    if kind in ("norm", "clip"):
        return _plain_grads(s)
    x = s["x"].detach()
    if kind == "quant":
        q = _round8(x.float(), c["tile"])
        qt = q.t() if c["tile"] == 128 else _round8(x.float().t(), 1)
        return q.to(x.dtype), qt.to(x.dtype)
    if kind == "linear":
        w = _unpacked(s["codes"], s["scales"], c["n"], c["k"])
        return (_round8(x.float(), 1) @ w.t()).to(x.dtype)
    x, dy, w = x.float(), s["dy"].float(), _round8(s["w"].detach(), 128)
    dw = _round8(dy.t(), 1) @ _round8(x.t(), 1).t()
    return (_round8(x, 1) @ w.t()).to(s["x"].dtype), (_round8(dy, 1) @ w).to(s["x"].dtype), dw


def _plain_sample(z, u, temperature, top_k, top_p, min_p):
    """In 64 bits: a token next to a border is another token.  Rows are taken in the order of falling logits, the lower index first."""
    t, v = z.shape
    row = lambda a: (a if torch.is_tensor(a) else torch.full((t,), a, dtype=torch.float32, device=z.device)).double()[:, None]
    heat, k, p, least = row(temperature), row(top_k), row(top_p), row(min_p)
    x = z.double()
    weight = torch.exp((x - x.amax(dim=1, keepdim=True)) / torch.where(heat > 0, heat, torch.ones_like(heat)))
    order = torch.sort(x, dim=1, descending=True, stable=True)[1]
    rank = torch.arange(v, device=z.device)[None, :]
    sorted_ = torch.gather(weight, 1, order)
    some = (rank < k) | (k <= 0)
    sorted_ = torch.where(some, sorted_, torch.zeros_like(sorted_))
    before = torch.cumsum(sorted_, dim=1) - sorted_
    keep = some & ((before < p * sorted_.sum(dim=1, keepdim=True)) | (p >= 1)) & (sorted_ >= least)
    keep = torch.where(heat > 0, keep | (rank == 0), rank == 0)
    weight = torch.where(torch.zeros_like(keep).scatter_(1, order, keep), weight, torch.zeros_like(weight))
    reached = torch.cumsum(weight, dim=1)
    total = reached[:, -1:]
    token = (reached <= u.double()[:, None] * total).sum(dim=1, keepdim=True)
    return token[:, 0], torch.log(torch.gather(weight, 1, token) / total)[:, 0].float()


def _plain_grads(s):
    c = s["case"]
    if c["most"]:
        norm = torch.stack([x.abs().max() for x in s["grads"]]).max().float()
    else:
        norm = torch.stack([x.double().square().sum() for x in s["grads"]]).sum().sqrt().float()
    norm = norm.reshape(1)
    if c["kind"] == "norm":
        return norm
    part = (c["limit"] / (norm + 1e-6)).clamp(max=1.0)
    return norm, torch.cat([(x.float() * part).to(x.dtype) for x in s["grads"]])


def _blocks(x, tile):
    """[blocks of rows, tile, blocks of columns, 128], filled up with zeros"""
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, -c % 128, 0, -r % tile))
    return x.view(-1, tile, x.shape[1] // 128, 128)


def _exponents(b):
    """of the least power of two that brings each block's largest element to at most 448 = 0.875 * 2^9"""
    top = b.abs().amax(dim=(1, 3), keepdim=True)
    m, e = torch.frexp(top)
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(top > 0, e, torch.full_like(e, -127)).clamp(min=-127)


def _two(e):
    """2^e exactly, which a power function need not be: e from -126 to 127"""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _e4m3(x):
    """To 4 significant bits, below 2^-6 to multiples of 2^-9; ties to even"""
    step = (torch.frexp(x)[1] - 1).clamp(min=-6) - 3
    return torch.round(x * _two(-step)) * _two(step)


def _round8(x, tile):
    """fp32 matrix -> the values that its 8-bit form stands for"""
    r, c = x.shape
    b = _blocks(x, tile)
    e = _exponents(b)
    b = torch.where(e > -127, _e4m3(b * _two(-e)) * _two(e.clamp(min=-126)), torch.zeros_like(b))
    return b.reshape(-1, b.shape[2] * 128)[:r, :c]


def _packed(x, tile):
    """codes and scales as a program keeps them"""
    r, _ = x.shape
    b = _blocks(x, tile)
    e = _exponents(b)
    codes = _e4m3(b * _two(-e)).reshape(-1, b.shape[2] * 128)[:r].to(torch.float8_e4m3fn).view(torch.uint8)
    scales = (e[:, 0, :, 0] + 127).to(torch.uint8)
    return codes.contiguous(), torch.nn.functional.pad(scales, (0, -scales.shape[1] % 4)).contiguous()


def _unpacked(codes, scales, r, c):
    power = torch.where(scales > 0, _two(scales.int() - 127), torch.zeros_like(scales, dtype=torch.float32))     # 0: a block of zeros
    power = power.repeat_interleave(128, dim=0)[:r].repeat_interleave(128, dim=1)[:, :codes.shape[1]]
    return (codes.view(torch.float8_e4m3fn).float() * power)[:, :c]


# ---- the same from the definitions in 64 bits ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "sample":
        return _exact_sample(case, s)
    if kind in ("norm", "clip"):
        total, most = 0.0, 0.0
        for x in s["flat"].split(1 << 28):
            total += float((x.double() ** 2).sum())
            most = max(most, float(x.abs().max()))
        norm = most if case["most"] else math.sqrt(total)
        if kind == "norm":
            return torch.tensor([norm], dtype=torch.float64)
        return torch.tensor([norm], dtype=torch.float64), s["flat"].double() * min(1.0, case["limit"] / (norm + 1e-6))
    x = s["x"].detach().double()
    if kind == "quant":
        return _exact8(x, case["tile"]), _exact8(x.t(), case["tile"])
    if kind == "linear":
        c = s["codes"].long()
        power, part = (c >> 3) & 15, (c & 7).double()
        w = torch.where(power > 0, (8 + part) * _power(power - 10), part * 2.0 ** -9) * torch.where(c > 127, -1.0, 1.0)
        i, j = torch.arange(case["n"], device=DEV) // 128, torch.arange(case["k"], device=DEV) // 128
        w = w[:, :case["k"]] * _power(s["scales"].long()[i][:, j] - 127)
        return _exact8(x, 1) @ w.t().contiguous()
    dy, w = s["dy"].double(), _exact8(s["w"].detach().double(), 128)
    y, dx = _exact8(x, 1) @ w.t().contiguous(), _exact8(dy, 1) @ w
    del w
    return y, dx, _exact8(dy.t(), 1) @ _exact8(x.t(), 1).t().contiguous()


def _power(e):
    table = torch.tensor([math.ldexp(1.0, i) for i in range(-300, 301)], dtype=torch.float64, device=e.device)
    return table[e.long() + 300]


def _floor_log2(a):
    """of positive numbers; the logarithm is only a first guess"""
    e = torch.floor(torch.log2(a)).long()
    return e - (a < _power(e)).long() + (a >= _power(e + 1)).long()


def _exact8(x, tile):
    """block by block, by logarithms"""
    r, c = x.shape
    out = torch.zeros(r, c, dtype=torch.float64, device=x.device)
    for j in range(0, c, 128):
        part = x[:, j:j + 128]
        top = part.abs().amax(dim=1)
        if tile > 1:
            rows = torch.arange(r, device=x.device) // tile
            top = torch.zeros(-(-r // tile), dtype=torch.float64, device=x.device).scatter_reduce_(0, rows, top, "amax")[rows]
        power = _floor_log2(torch.where(top > 0, top, torch.ones_like(top))) - 8
        power = torch.where(top > 448 * _power(power), power + 1, power)
        scale = _power(power.clamp(min=-127))[:, None]
        a = part.abs() / scale
        grid = _power(_floor_log2(a.clamp(min=2.0 ** -6)) - 3)
        out[:, j:j + 128] = torch.sign(part) * torch.round(a / grid) * grid * scale
    return out


def _exact_sample(case, s):
    if case["t"] * case["v"] > 1 << 27:
        return None
    t = case["t"]
    value = lambda key: s[key].double().cpu().numpy() if torch.is_tensor(s[key]) else np.full(t, np.float32(s[key]), np.float64)
    heat, k, p, least, u = value("temperature"), value("top_k"), value("top_p"), value("min_p"), s["u"].double().cpu().numpy()
    z = s["z"].double().cpu().numpy()
    said = np.zeros(t)
    for i in range(t):
        if heat[i] == 0:
            continue
        order = np.argsort(-z[i], kind="stable")
        if k[i] > 0:
            order = order[:int(k[i])]
        w = np.exp((z[i, order] - z[i, order[0]]) / heat[i])
        count = len(order)
        if p[i] < 1:
            count = min(count, int(np.searchsorted(np.cumsum(w), p[i] * w.sum(), side="left")) + 1)
        count = max(1, min(count, int((w >= least[i]).sum())))
        places = np.sort(order[:count])
        w = np.exp((z[i, places] - z[i, order[0]]) / heat[i])
        reached = np.cumsum(w)
        said[i] = math.log(w[int(np.searchsorted(reached, u[i] * reached[-1], side="right"))] / reached[-1])
    return None, torch.from_numpy(said)
