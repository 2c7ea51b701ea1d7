"""float64 oracle for the norms of query and key heads.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): the product path never
imports this module.
"""
from __future__ import annotations

import numpy as np


def head_norm(x, weight, eps: float) -> np.ndarray:
    """x [T, heads, dim], each head divided by the root of its mean square (and eps), times weight [dim] or None."""
    x = np.asarray(x, dtype=np.float64)
    y = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
    return y if weight is None else y * np.asarray(weight, dtype=np.float64)
