"""Tokens drawn from logits of any leading dimensions, over lpmm_sample.  Orchestration only -- every number but the random ones is
computed by lpmm4.so.

    tokens, logprob = sample(logits, temperature=0.8, top_p=0.95)
"""
from __future__ import annotations

import torch

from . import binding as _b
from .w4 import _flat


def sample(logits: torch.Tensor, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u: torch.Tensor = None, generator: torch.Generator = None):
    """(tokens, logprob), shaped like logits (..., vocabulary) without the last dimension: a token drawn from each distribution and the logarithm of the probability it
    was drawn with.  temperature 0 takes the largest logit; top_k (0: all), top_p and min_p as in lpmm4.h; each a number, or a tensor (float32;
    top_k int32) of the leading dimensions.  u: random numbers from [0, 1), float32, of the leading dimensions; drawn with `generator` if not given."""
    lead = logits.shape[:-1]
    if u is None:
        u = torch.rand(lead, dtype=torch.float32, device=logits.device, generator=generator)
    elif u.shape != lead:
        raise ValueError(f"sample: u must be {tuple(lead)}, like the logits")

    def each(x, name):
        if not torch.is_tensor(x):
            return x
        if x.shape != lead:
            raise ValueError(f"sample: {name} must be a number or {tuple(lead)}, like the logits")
        return x.reshape(-1).contiguous()

    tokens, logprob = _b.lpmm_sample(_flat(logits.detach(), logits.shape[-1]), u.reshape(-1).contiguous(), each(temperature, "temperature"), each(top_k, "top_k"),
                                     each(top_p, "top_p"), each(min_p, "min_p"))
    return tokens.view(lead), logprob.view(lead)
