"""Adapters' inner sums next to the largest fp32 numbers, and infinite weights."""
import numpy as np
import pytest
import torch

from test_gpu_adapter import Call, ppas  # noqa: F401

pytestmark = pytest.mark.gpu

# units, tiles of 128 rows, tiles of 64 rows
STEPS = [([1, 1, 20], [0, 1, 0], 320, [72, 40], 16), ([1, 150, 470], [1, 0, 1], 320, [136, 40], 16),
         ([300, 100, 77, 129, 1], [0, 1, 0, 2, -1], 2048, [1024, 264], 64)]


@pytest.mark.parametrize("lens,ids,hidden,slices,rank", STEPS)
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_sums_past_the_largest_bf16(ppas, lens, ids, hidden, slices, rank, sign):  # noqa: F811
    """An inner sum between the largest bf16 number and the largest fp32 one is finite, and so is what it adds."""
    c = Call(lens, ids, hidden, slices, rank, seed=1)
    most = float(torch.finfo(torch.bfloat16).max)
    c.x[:] = 0
    c.x[:, 0], c.x[:, 9] = sign * most, sign * 1.5 * 2.0 ** 119  # 3/4 of the largest ones' step of 2^120
    c.a.zero_()
    c.a[:, 3, 0] = c.a[:, 3, 9] = 1.0
    c.b.mul_(2.0 ** -120)
    ppas.ppas_adapter_add(**c.args())
    c.check()


@pytest.mark.parametrize("lens,ids,hidden,slices,rank", STEPS)
def test_an_infinite_sum_is_infinite(ppas, lens, ids, hidden, slices, rank):  # noqa: F811
    """x with an infinity times positive weights: that row alone is infinite, not a NaN."""
    c = Call(lens, ids, hidden, slices, rank, seed=2, scales=False)
    c.a.abs_().add_(0.01)
    c.b.abs_().add_(0.01)
    clean = c.out.clone()
    ppas.ppas_adapter_add(**c.args(out=clean))
    c.x[4, 3] = float("inf")
    ppas.ppas_adapter_add(**c.args())
    torch.cuda.synchronize()
    same = torch.ones(c.T, dtype=torch.bool, device="cuda")
    same[4] = False
    assert torch.equal(c.out[same], clean[same])
    assert bool((c.out[4] == float("inf")).all())


@pytest.mark.parametrize("lens,ids,hidden,slices,rank", STEPS)
def test_an_infinite_weight_stays_in_its_column(ppas, lens, ids, hidden, slices, rank):  # noqa: F811
    """A row of B with an infinity spoils that column of its adapter's rows, nothing else."""
    c = Call(lens, ids, hidden, slices, rank, seed=3)
    clean = c.out.clone()
    ppas.ppas_adapter_add(**c.args(out=clean))
    c.b[1, 5, 2] = float("inf")
    ppas.ppas_adapter_add(**c.args())
    torch.cuda.synchronize()
    rows = torch.from_numpy(np.repeat(c.ids, c.lens) == 1).cuda()
    same = torch.ones_like(c.out, dtype=torch.bool)
    same[rows, 5] = False
    assert torch.equal(c.out[same], clean[same])
    assert not bool(c.out[rows, 5].isfinite().any())
