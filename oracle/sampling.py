"""float64 oracle for sampling with temperature, top-k, top-p and min-p.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): the product path never
imports this module.

What is computed
----------------
One row of logits at a time, from the definition: probabilities ``p_i``
proportional to ``exp(x_i / T)``, tokens in descending order of their logits (the
lower index first among equals); the first ``top_k``; of these the fewest whose
probabilities reach ``top_p`` of theirs; of these the ones with at least ``min_p``
of the largest probability; and the token at which the running sum passes
``u`` times the sum of what is kept.

A draw within a rounding of the edge of two tokens, and a cut within a rounding
of its target, may fall either way in 32 bits, so ``accepts`` takes a relative
tolerance on running sums and says whether a token and its log-probability are
among the answers that it allows.
"""
from __future__ import annotations

import numpy as np


def candidates(x, temperature: float):
    """(token order, weights in that order): weights exp((x - max) / T), 0 for -inf and NaN."""
    x = np.asarray(x, dtype=np.float64).copy()
    x[np.isnan(x)] = -np.inf
    order = np.argsort(-x, kind="stable")
    top = x[order[0]]
    w = np.zeros_like(x)
    if top == np.inf:
        w[x == np.inf] = 1.0
    elif top > -np.inf:
        w = np.exp((x - top) / temperature)
    return order, w[order]


def kept_weight(w, top_k: int, top_p: float, min_p: float):
    """Running sum at the last kept token, and their count."""
    n = len(w)
    if 0 < top_k < n:
        n = top_k
    cum = np.cumsum(w)
    if top_p < 1:
        n = min(n, int(np.searchsorted(cum, top_p * cum[n - 1], side="left")) + 1)
    if min_p > 0:
        n = max(1, min(n, int(np.count_nonzero(w >= min_p))))
    return cum[n - 1], n


def sample(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """(token, logprob) by the definition."""
    order, w = candidates(x, temperature if temperature > 0 else 1.0)
    if w.sum() == 0:
        return -1, -np.inf
    if not temperature > 0:
        return int(order[0]), 0.0
    total, n = kept_weight(w, top_k, top_p, min_p)
    at = min(int(np.searchsorted(np.cumsum(w), u * total, side="right")), n - 1)
    return int(order[at]), float(np.log(w[at] / total))


def accepts(token, logprob, x, temperature, top_k, top_p, min_p, u, tol):
    """Whether (token, logprob) is an answer when running sums and the products
    with top_p, min_p and u are only known to a relative ``tol``."""
    want = sample(x, temperature, top_k, top_p, min_p, u)
    if not temperature > 0 or want[0] < 0:
        return (int(token), float(logprob)) == want
    order, w = candidates(x, temperature)
    cum = np.cumsum(w)
    low, n_low = kept_weight(w, top_k, top_p * (1 - tol) if top_p < 1 else top_p, min_p * (1 + tol))
    high, n_high = kept_weight(w, top_k, min(top_p * (1 + tol), 1 - 1e-15) if top_p < 1 else top_p, min_p * (1 - tol))
    at = int(np.nonzero(order == token)[0][0])
    if at >= n_high or w[at] == 0:
        return False
    first, last = cum[at] - w[at], cum[at]
    if u * low > last + tol * high or u * high < first - tol * high:
        return False
    return np.log(w[at] / high) - 2 * tol <= logprob <= min(0.0, np.log(w[at] / low)) + 2 * tol
