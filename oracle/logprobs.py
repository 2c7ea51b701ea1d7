"""float64 oracle for log probabilities of tokens, entropy and alternatives.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): the product path never
imports this module.
"""
from __future__ import annotations

import numpy as np


def row(x, given: int, n_top: int, largest: float):
    """(log p of the given token, entropy, top tokens, their log p) of one row of logits."""
    x = np.asarray(x, dtype=np.float64).copy()
    x[np.isnan(x)] = -np.inf
    x = np.minimum(x, largest)
    top_tokens, top_logprobs = np.full(n_top, -1, np.int64), np.full(n_top, -np.inf)
    m = x.max()
    if m == -np.inf:
        return (0.0 if given < 0 else -np.inf), 0.0, top_tokens, top_logprobs
    lp = x - m - np.log(np.sum(np.exp(x - m)))
    p = np.exp(lp)
    entropy = -np.sum(p[p > 0] * lp[p > 0])
    order = np.argsort(-x, kind="stable")[:n_top]
    order = order[x[order] > -np.inf]
    top_tokens[:len(order)], top_logprobs[:len(order)] = order, lp[order]
    return (0.0 if given < 0 else lp[given] if given < len(x) else -np.inf), entropy, top_tokens, top_logprobs
