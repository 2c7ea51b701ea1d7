"""float64 oracle for low-rank adapters beside a shared projection.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): the product path never
imports this module.
"""
from __future__ import annotations

import numpy as np


def adapter_add(x, y, q_lens, adapters, a, b, scales, slice_cols, rank: int) -> np.ndarray:
    """x [T, hidden], y [T, cols], a [n, slices * rank, hidden], b [n, cols, rank], scales [n] or None."""
    return y + _delta(x, q_lens, adapters, a, b, scales, slice_cols, rank)


def bound(x, y, q_lens, adapters, a, b, scales, slice_cols, rank: int) -> np.ndarray:
    """What a result in bf16 from fp32 sums may be off by: half a step of the result
    (2^-8 of it); of the inner sums one rounding of 2^-23 for each 16 terms and 20
    more of the joins, relative to the sum of the terms' sizes, and 2^-17 of
    their own size for the two bf16 numbers that stand for them; of the outer sums
    a rounding for each 8 terms (two products for every 16) and 4 more."""
    hidden = x.shape[1]
    inner = (hidden / 16 + 20) * 2.0 ** -23 + 2.0 ** -17
    outer = (rank / 8 + 4) * 2.0 ** -23
    size = _delta(np.abs(x), q_lens, adapters, np.abs(a), np.abs(b), None if scales is None else np.abs(scales),
                  slice_cols, rank)
    return 2.0 ** -8 * np.abs(adapter_add(x, y, q_lens, adapters, a, b, scales, slice_cols, rank)) + \
        (inner + outer) * size + 1e-37


def _delta(x, q_lens, adapters, a, b, scales, slice_cols, rank):
    out = np.zeros((x.shape[0], int(np.sum(slice_cols))))
    at = 0
    for n, which in zip(q_lens, adapters):
        if which >= 0:
            inner = x[at:at + n] @ a[which].T
            c = 0
            for j, cols in enumerate(slice_cols):
                delta = inner[:, j * rank:(j + 1) * rank] @ b[which, c:c + cols].T
                out[at:at + n, c:c + cols] = delta * (1.0 if scales is None else scales[which])
                c += cols
        at += n
    return out
