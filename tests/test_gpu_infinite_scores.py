"""Scores of -inf on the GPU (queries and keys whose products pass the range of
fp32): such a key has weight 0, wherever it lies in a row's context, as in the
float64 oracle.  Shared prefixes (prefix pieces, own keys, their join) and the
ordinary step (decode rows and prompt chunks).

Tolerance: that of the attention tests, 5e-3 of the result's norm and 2e-2 an
element; a weight of 0 is exact."""
import numpy as np
import pytest
import torch

from _cases import MAX_ABS, host64
from oracle import attention as oa
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


@pytest.mark.parametrize("lo,hi", [(0, 16), (0, 150), (100, 290), (0, 290)])
@pytest.mark.parametrize("hq,hk", [(16, 2), (8, 8), (32, 8)])
def test_ordinary_step(ppas, hq, hk, lo, hi):  # noqa: F811
    """Decode rows (a few, in clusters; and enough to fill the device) and a chunk of 40 tokens."""
    for n, q_len in ((2, 1), (70, 1), (2, 40)):
        b = Batch(hq, hk, [1] * n, [0] * n, [300 + 7 * (r % 5) for r in range(n)], seed=3)
        if q_len > 1:
            g = torch.Generator(device="cuda")
            g.manual_seed(4)
            b.q = torch.randn((n * q_len, hq, 128), generator=g, device="cuda").to(torch.bfloat16)
        # (a chunk's first token sees 261 keys at least)
        _sink(b, range(n), lo, min(hi, 255) if q_len > 1 else hi)
        lens = [q_len] * n
        size = ppas.ppas_attention_workspace_size(lens, b.ctx, hq, hk)
        ws = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
        out = torch.empty((n * q_len, hq, 128), dtype=torch.bfloat16, device="cuda")
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        ppas.ppas_attention_step(b.q, b.k, b.v, b.blocks, b.d_table, b.width, lens, b.ctx, hq, hk, 128, 128 ** -0.5,
                                 out, False, ws, size, err)
        torch.cuda.synchronize()
        assert int(err.item()) == 0
        k, v = (torch.nan_to_num(x, nan=0.0) for x in (b.k, b.v))
        got = host64(out)
        want = oa.paged_attention(host64(b.q), host64(k), host64(v), b.table, lens, b.ctx, 128 ** -0.5)
        assert np.all(np.isfinite(got))
        assert np.abs(got - want).max() <= MAX_ABS and np.linalg.norm(got - want) <= 5e-3 * np.linalg.norm(want)
