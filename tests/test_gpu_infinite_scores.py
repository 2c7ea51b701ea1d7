"""Scores of -inf on the GPU (queries and keys whose products pass the range of
fp32): such a key has weight 0, wherever it lies in a row's context, as in the
float64 oracle.

Tolerance: that of the attention tests, 5e-3 of the result's norm and 2e-2 an
element; a weight of 0 is exact."""
import pytest
import torch

from test_gpu_shared_attention import Batch, ppas  # noqa: F401

pytestmark = pytest.mark.gpu


def _sink(b, rows, lo, hi):
    """Keys lo .. hi - 1 of these rows get a score of -1e40 / sqrt(128) or so."""
    b.q[..., 0] = 1e20
    b.k[..., 0] = torch.where(torch.isnan(b.k[..., 0]), b.k[..., 0], torch.zeros_like(b.k[..., 0]))
    for r in rows:
        for j in range(lo, min(hi, b.ctx[r])):
            b.k[int(b.table[r, j // 16]), :, j % 16, 0] = -1e20


@pytest.mark.parametrize("lo,hi", [(0, 16), (0, 64), (0, 5), (16, 48), (40, 79), (3, 300)])
@pytest.mark.parametrize("hq,hk", [(16, 2), (8, 8)])
def test_own_keys_without_weight(ppas, hq, hk, lo, hi):  # noqa: F811
    b = Batch(hq, hk, [3], [0], [80, 333, 1000], seed=1)
    _sink(b, [0, 1, 2], lo, min(hi, 79))
    b.check(b.call(ppas))


@pytest.mark.parametrize("lo,hi", [(0, 128), (0, 640), (100, 400), (512, 720), (640, 656), (0, 656)])
@pytest.mark.parametrize("hq,hk,rows", [(16, 2, 20), (8, 8, 40)])
def test_prefix_keys_without_weight(ppas, hq, hk, rows, lo, hi):  # noqa: F811
    b = Batch(hq, hk, [rows], [640], [100] * rows, seed=2)
    _sink(b, range(rows), lo, hi)
    b.check(b.call(ppas))
