"""Sampling from rows with +inf logits on the GPU: such a logit counts as the
largest finite value of the logits' type, so any number of them are ties that go
by index, in every path a row can take (few ties, hundreds, whole vocabularies).

The tokens are exact: every tied weight is 2^40, all others are 0, so with m
tokens kept S = m 2^40 and the draw is tie floor(u S) / 2^40.  Log-probabilities
are -ln m to fp32 (1e-6 of max(1, ln m))."""
import math

import numpy as np
import pytest
import torch

from test_gpu_sample import _call, ppas  # noqa: F401

pytestmark = pytest.mark.gpu
LARGEST = {False: 3.4028234663852886e38, True: 3.3895313892515355e38}
UNIT = 1 << 40
RULES = [(1.0, "all", 1.0, 0.0), (0.7, "half", 1.0, 0.0), (1.0, "all", 0.6, 0.0), (1.3, "half", 0.5, 0.3),
         (1e-3, "one", 1.0, 0.0), (1e6, "all", 0.99, 0.9), (2.0, "more", 0.25, 0.0), (0.0, "all", 1.0, 0.0)]
U = [0.0, 0.5, 0.999, 1 - 2.0 ** -24, 0.3, 0.77, 0.9, 0.6]


def _want(ties, rule, u):
    """(index, kept ties) of the tokens at `ties`, in the order of their indexes."""
    t, k, p, _ = rule
    m = len(ties)
    if t <= 0:
        return ties[0], 1
    keep = {"all": m, "more": m, "half": m // 2 + 1, "one": 1}[k]
    keep = min(keep, m)
    if p < 1:
        keep = min(keep, -(-math.ceil(float(np.float32(p)) * float(keep * UNIT)) // UNIT))
    at = min(int(float(np.float32(u)) * float(keep * UNIT)), keep * UNIT - 1)
    return ties[at // UNIT], keep


def _top_k(rule, m):
    return {"all": 0, "half": m // 2 + 1, "one": 1, "more": m + 3}[rule[1]]


def _check(ppas, x, ties):  # noqa: F811
    n = x.shape[0]
    rules = [RULES[r % len(RULES)] for r in range(n)]
    u = np.array([U[(r * 3) % len(U)] for r in range(n)], np.float32)
    tokens, lp = _call(ppas, x, [r[0] for r in rules], [_top_k(r, len(t)) for r, t in zip(rules, ties)],
                       [r[2] for r in rules], [r[3] for r in rules], u)
    for r in range(n):
        token, kept = _want(ties[r], rules[r], u[r])
        assert tokens[r] == token, (r, rules[r], len(ties[r]))
        assert abs(lp[r] + math.log(kept)) <= 1e-6 * max(1.0, math.log(kept)), (r, rules[r], len(ties[r]))


def _rows(n, v, counts, bf16, mixed, seed):
    """[n, v] logits, the +inf places of each row; `mixed`: every other tie is the largest finite value."""
    g = np.random.default_rng(seed)
    x = g.normal(0, 3, (n, v)).astype(np.float32)
    x[:, ::97] = -math.inf
    x[:, 5::101] = math.nan
    ties = []
    for r in range(n):
        at = np.sort(g.permutation(v)[:counts[r % len(counts)]])
        x[r, at] = math.inf
        if mixed:
            x[r, at[::2]] = LARGEST[bf16]
        ties.append(at.tolist())
    y = torch.from_numpy(x).cuda()
    return (y.to(torch.bfloat16) if bf16 else y), ties


@pytest.mark.parametrize("mixed", [False, True])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("count", [1, 2, 127, 128, 129, 511, 512, 513, 1023, 1024, 1025, 3000, 20000])
def test_numbers_of_infinities(ppas, count, bf16, mixed):  # noqa: F811
    x, ties = _rows(16, 20000, [count], bf16, mixed, count)
    _check(ppas, x, ties)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,v", [(2, 262144), (3, 7), (40, 1000), (8, 152000)])
def test_whole_vocabularies_of_infinities(ppas, n, v, bf16):  # noqa: F811
    x = torch.full((n, v), math.inf, device="cuda", dtype=torch.bfloat16 if bf16 else torch.float32)
    _check(ppas, x, [list(range(v))] * n)


@pytest.mark.parametrize("bf16", [False, True])
def test_rows_too_long_for_shared_memory(ppas, bf16):  # noqa: F811
    x, ties = _rows(312, 90000, [1, 100, 200, 700, 1500, 30000, 2, 5000], bf16, False, 9)
    _check(ppas, x, ties)


@pytest.mark.parametrize("bf16", [False, True])
def test_largest_finite_value_ties_with_infinity(ppas, bf16):  # noqa: F811
    """The largest logit, temperature 0: the lowest index of both kinds."""
    x = torch.zeros((2, 9), device="cuda")
    x[0, 4], x[0, 6] = LARGEST[bf16], math.inf
    x[1, 4], x[1, 6] = math.inf, LARGEST[bf16]
    x = x.to(torch.bfloat16) if bf16 else x
    tokens, lp = _call(ppas, x, 0.0)
    assert list(tokens) == [4, 4] and list(lp) == [0.0, 0.0]
