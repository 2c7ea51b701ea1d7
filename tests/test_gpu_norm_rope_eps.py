"""Head norms whose eps is next to either end of the fp32 range, so that the squares of
the values it is added to leave that range, below or above, every element against the
float64 oracle (tolerance: that of ``test_gpu_norm_rope``; a sum is taken again times a
power of two where squares are lost, which rounds nothing)."""
import pytest
import torch

from test_gpu_norm_rope import Step, ppas  # noqa: F401

pytestmark = pytest.mark.gpu


# values next to the root of eps and on both sides of it; 2^-100 = 7.9e-31 and 2^100 = 1.3e30 are where
# other sums are looked at, 2^-55 = 2.8e-17 the root of 2^-110
@pytest.mark.parametrize("gain,eps", [
    (1e-23, 1e-45), (1e-21, 1e-45), (3e-20, 1e-40), (1e-38, 1e-45), (0.0, 1e-45), (1e-38, 1e-38), (1e-16, 1e-32),
    (2.5e-18, 1e-45), (2.4e-17, 1e-35), (1e-15, 7.8e-31), (1e-15, 8e-31), (1e-22, 7.8e-31), (1.0, 1e-45), (1e30, 1e-45),
    (3e18, 1e38), (1e19, 1e38), (1.2e18, 3.4e38), (1e19, 3.4e38), (1e15, 1.2e30), (1e15, 1.3e30), (1e30, 1e38), (1.0, 3.4e38),
    (1e-30, 1e38), (0.0, 1e38)])
@pytest.mark.parametrize("D,inter,shift", [(128, False, 0), (128, True, 0), (80, False, 0), (128, False, 1)])
def test_values_next_to_the_root_of_eps(ppas, gain, eps, D, inter, shift):  # noqa: F811
    s = Step(20, 4, 2, D, D, inter, seed=3, gain=gain, eps=eps, shift=shift)
    ppas.ppas_norm_rope_append(**s.args())
    s.check()


@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1e-6, 1e38])
@pytest.mark.parametrize("D,shift", [(128, 0), (80, 0), (128, 1)])
def test_heads_of_all_sizes_side_by_side(ppas, eps, D, shift):  # noqa: F811
    """Heads of one warp whose sums are in range, lost below and past it above."""
    s = Step(33, 8, 4, D, 64, False, seed=4, eps=eps, shift=shift)
    for i, gain in enumerate((1e-38, 1e-23, 0.0, 1e-18, 1.0, 1e18, 1e19, 1e37)):
        s.q[:, i] *= gain
        s.q[i + 8] = s.q[i + 8].flip(0)
    for i, gain in enumerate((1e-22, 1e19, 1.0, 0.0)):
        s.k[:, i] *= gain
    ppas.ppas_norm_rope_append(**s.args())
    s.check()


def test_a_nan_stays_in_its_head(ppas):  # noqa: F811
    for eps in (1e-45, 1e38):
        s, clean = (Step(9, 4, 2, 128, 128, False, seed=7, eps=eps, gain=1e-23) for _ in range(2))
        s.q[3, 1, 5], s.q[4, 2, 7] = float("nan"), float("inf")
        for x in (s, clean):
            ppas.ppas_norm_rope_append(**x.args())
        torch.cuda.synchronize()
        same = torch.ones(9, 4, dtype=torch.bool)
        same[3, 1] = same[4, 2] = False
        assert torch.equal(s.out[:9][same.cuda()], clean.out[:9][same.cuda()]) and torch.equal(s.kc, clean.kc)
        assert bool(s.out[3, 1].isnan().all()) and bool(s.out[4, 2, [7, 71]].isnan().all())
