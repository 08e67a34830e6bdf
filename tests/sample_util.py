"""The plain 64-bit form of drawing tokens, row by row on the CPU, written from the formulas in include/lpmm4.h."""
import math

import numpy as np
import torch


def draw(z, u, temperature, top_k, top_p, min_p):
    """One row (CPU tensor) -> (token, logprob, how near the draw is to another outcome: in weights, whose largest is 1; the sum of all weights)"""
    x = z.double().numpy()
    top = x.max() if not np.isnan(x).any() else math.nan
    if not top > -math.inf:
        return -1, math.nan, math.inf, 1.0
    order = np.argsort(-x, kind="stable")
    if not temperature > 0:
        return int(order[0]), 0.0, math.inf, 1.0
    with np.errstate(invalid="ignore"):
        w = np.where(x == top, 1.0, np.where(np.isneginf(x) | np.isposinf(top), 0.0, np.exp((x - top) / temperature)))
    near = math.inf
    n = len(x)
    if 0 < top_k < n:
        n = top_k
    if top_p < 1:
        sums = np.cumsum(w[order[:n]])
        before = np.concatenate([[0.0], sums[:-1]])
        border = top_p * sums[-1]
        near = min(near, float(np.abs(before[1:] - border).min())) if n > 1 else near
        n = max(1, int((before < border).sum()))
    if min_p > 0:
        n = max(1, min(n, int((w[order] >= min_p).sum())))
    kept = np.sort(order[:n])
    sums = np.cumsum(w[kept])
    at = max(float(u) if u == u else 0.0, 0.0) * sums[-1]
    i = int(np.searchsorted(sums, at, side="right"))
    if i >= n or at >= sums[-1]:
        i = int(np.searchsorted(sums, sums[-1], side="left"))
    elif at > 0:
        near = min(near, float(np.abs(sums - at).min()))
    token = int(kept[i])
    d = 0.0 if x[token] == top else (x[token] - top) / temperature
    return token, d - math.log(sums[-1]), near, float(w.sum())


def check(z, u, temperature, top_k, top_p, min_p, tokens, logprob, what, unsure=0):
    """Weights, the largest of them 1, are whole numbers of 2^-46 and their sums exact: a border can move by v 2^-47, and by v 2^-53 of the sum for the
    64-bit sums here; a draw nearer to one than 4 times that may fall on the other side: `unsure` rows at most,
    which are passed over (none, unless a test says so).  The logarithm is rounded to fp32 once."""
    t, v = z.shape
    of = lambda o, r: float(o[r]) if torch.is_tensor(o) else float(np.float32(o))
    tokens, logprob = tokens.cpu(), logprob.cpu().double()
    for r in range(t):
        k = int(top_k[r]) if torch.is_tensor(top_k) else top_k
        token, lp, near, size = draw(z[r], of(u, r), of(temperature, r), k, of(top_p, r), of(min_p, r))
        equal = bool(((z[r] == z[r].max()) | (z[r] == -math.inf)).all())          # weights of 1 and 0: nothing is rounded, and no border moves
        if not (equal or near > v * (2.0 ** -45 + size * 2.0 ** -51)):
            assert unsure > 0, f"{what}, row {r}: another seed is needed"
            unsure -= 1
            continue
        assert int(tokens[r]) == token, f"{what}, row {r}: token {int(tokens[r])}, not {token}"
        if math.isnan(lp):
            assert math.isnan(float(logprob[r])), f"{what}, row {r}"
        else:
            assert abs(float(logprob[r]) - lp) <= 2.0 ** -24 * abs(lp) + v * 2.0 ** -44, f"{what}, row {r}: {float(logprob[r])}, not {lp}"
