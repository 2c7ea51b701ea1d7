"""float64 oracle for rotary positions and the append of rotated keys.

TEST INFRASTRUCTURE ONLY (see ``oracle/__init__.py``): the product path never
imports this module.

What is computed
----------------
Pair ``i`` of a head at position ``t`` is a complex number that turns by
``t f_i`` and is scaled by ``factor``; the half layout pairs ``x[i]`` with
``x[i + r/2]``, the interleaved one ``x[2i]`` with ``x[2i + 1]``, and values from
``r`` on are left alone.  Arithmetic is float64 on the widened inputs.
"""
from __future__ import annotations

import math

import numpy as np


def rotate(x: np.ndarray, positions, inv_freq, rotary: int, interleaved: bool, factor: float = 1.0) -> np.ndarray:
    """x [T, heads, dim] at positions [T]; inv_freq [rotary / 2]."""
    x = np.asarray(x, dtype=np.float64)
    angle = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float64)[None, :]
    turn = factor * np.exp(1j * angle)[:, None, :]
    out = x.copy()
    if interleaved:
        z = (x[..., 0:rotary:2] + 1j * x[..., 1:rotary:2]) * turn
        out[..., 0:rotary:2], out[..., 1:rotary:2] = z.real, z.imag
    else:
        z = (x[..., :rotary // 2] + 1j * x[..., rotary // 2:rotary]) * turn
        out[..., :rotary // 2], out[..., rotary // 2:rotary] = z.real, z.imag
    return out


def frequencies(kind: str, rotary: int, base: float, scale: float = 1.0, original: int = 0, low: float = 1.0,
                high: float = 4.0):
    """(inverse frequencies, factor), written out from the definitions one index at a time."""
    if kind == "base":
        base = base * scale ** (rotary / (rotary - 2))
    f = [base ** (-2 * i / rotary) for i in range(rotary // 2)]
    if kind == "linear":
        return [x / scale for x in f], 1.0
    if kind == "bands":
        out = []
        for x in f:
            turns = original / (2 * math.pi / x)
            if turns >= high:
                out.append(x)
            elif turns <= low:
                out.append(x / scale)
            else:
                blend = (turns - low) / (high - low)
                out.append((1 - blend) * x / scale + blend * x)
        return out, 1.0
    if kind == "ramp":
        def index(turns):
            return rotary * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
        a, b = max(math.floor(index(high)), 0), min(math.ceil(index(low)), rotary - 1)
        b = b if b > a else a + 0.001
        out = []
        for i, x in enumerate(f):
            share = min(max((i - a) / (b - a), 0.0), 1.0)
            out.append(x / scale * share + x * (1 - share))
        return out, 0.1 * math.log(scale) + 1.0
    return f, 1.0
