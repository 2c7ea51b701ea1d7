"""Rotary angles of any finite frequency on the GPU, from the smallest to the
largest fp32 number, at positions over all of int32, against exact arithmetic:
position * frequency is a rational number, reduced modulo 2 pi with pi to 600 bits.

Tolerance: as for the append itself, one rounding to bf16 (2^-8 relative) of an
fp32 result whose angle is off by at most 2^-25 turn, 1e-6 of |a| + |b|."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from paper_2608_15171_gb300 import workloads as wl
from test_gpu_rope import ppas  # noqa: F401

pytestmark = pytest.mark.gpu
BITS = 600


def _arctan_inverse(n, bits):
    """floor of 2^bits arctan(1 / n), to some units."""
    total, term, k = 0, (1 << bits) // n, 1
    while term:
        total += term // k if k % 4 == 1 else -(term // k)
        term //= n * n
        k += 2
    return total


PI = Fraction(4 * (4 * _arctan_inverse(5, BITS) - _arctan_inverse(239, BITS)), 1 << BITS)


def _angle(position, f):
    """position * f modulo 2 pi, in [-pi, pi], as a double."""
    x = Fraction(int(position)) * Fraction(float(f))
    turns = x / (2 * PI)
    return float((turns - round(turns)) * 2 * PI)


def test_reduction():
    for p, f in ((1, 0.5), (3, 1.0), (100000, 0.25), (-7, 0.75)):
        assert abs(math.remainder(p * f, 2 * math.pi) - _angle(p, f)) < 1e-9
    assert abs(float(PI) - math.pi) < 1e-15


FREQUENCIES = [0.3, 1.0, 255.7, 65537.25, 16777213.0, 2.0 ** 24, 33554434.0, 123456789.0, 2.0 ** 33, 1e10, -3e12, 1e15,
               2.0 ** 47, 1e18, 2.0 ** 63, 2.0 ** 64, 1e20, -1e25, 2.0 ** 87, 2.0 ** 88, 1e30, 1e35,
               3.4028234663852886e38, -3.0e38, 1e-38, 1e-45, -1e-7, 0.0, 6.2831855, 1e4, 1e7, 3.0]


@pytest.mark.parametrize("shift", [0, 1])  # 16-byte rows, and the kernel for any alignment
@pytest.mark.parametrize("interleaved", [False, True])
def test_every_finite_frequency(ppas, interleaved, shift):  # noqa: F811
    half, hk, dim = len(FREQUENCIES), 1, 2 * len(FREQUENCIES)
    f = np.array(FREQUENCIES, np.float32)
    pos = np.array([0, 1, -1, 2, 3, 1000, 131071, -131072, 10 ** 6 + 3, 10 ** 9 + 7, 2 ** 31 - 1, -2 ** 31], np.int32)
    t = len(pos)
    row = hk * dim + shift
    k = wl.bf16_normal((t * row + 8,), 3, "cuda")[shift:].as_strided((t, hk, dim), (row, dim, 1))
    v = k.clone().contiguous()
    blocks = 1
    kc = torch.zeros((blocks, hk, 16, dim), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ppas.ppas_rope_append(None, k, v, 0, row, hk * dim, torch.from_numpy(pos).cuda(),
                          torch.arange(t, dtype=torch.int32, device="cuda"), t, torch.from_numpy(f).cuda(), dim,
                          interleaved, 1.0, None, kc, vc, blocks, 0, hk, dim, err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    got = kc[0, 0, :t].double().cpu().numpy()
    x = k[:, 0].double().cpu().numpy()
    angle = np.array([[_angle(p, y) for y in f] for p in pos])
    a, b = (x[:, 0::2], x[:, 1::2]) if interleaved else (x[:, :half], x[:, half:])
    ga, gb = (got[:, 0::2], got[:, 1::2]) if interleaved else (got[:, :half], got[:, half:])
    size = np.abs(a) + np.abs(b)
    for have, want in ((ga, a * np.cos(angle) - b * np.sin(angle)), (gb, b * np.cos(angle) + a * np.sin(angle))):
        off = np.abs(have - want) - (2.0 ** -8 * np.abs(want) + 1e-6 * size)
        bad = np.unravel_index(off.argmax(), off.shape)
        assert off.max() <= 0, (pos[bad[0]], f[bad[1]], off.max())
