"""Log probabilities of rows masked with finite constants, against the float64 oracle, and
what a row's answers have to do with the rows beside it (tolerances: ``test_gpu_logprobs``)."""
import numpy as np
import pytest
import torch

from test_gpu_logprobs import _call, _check, _logits, ppas  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mask", [-1e3, -2.9e6, -3e6, -1e7, -1e9, -1e10, -6e29, -8e29, -1e30, -2e30, -3e38])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,v", [(6, 5001), (2, 152000), (700, 3001)])
def test_finite_masks(ppas, mask, dtype, n, v):  # noqa: F811
    """A few, most and all but a few of the logits masked, all of them, one half of the row, in runs and apart."""
    x = _logits(n, v, seed=v, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(3)
    part = torch.rand((n, v), generator=g, device="cuda")
    kind = torch.arange(n, device="cuda")[:, None] % 6
    column = torch.arange(v, device="cuda")[None]
    masked = torch.where(kind == 0, part < 0.01, torch.where(kind == 1, part < 0.9, torch.where(
        kind == 2, column % 997 != 5, torch.where(kind == 3, column >= 0, torch.where(
            kind == 4, column < v // 2, column // 64 % 3 > 0)))))
    x = torch.where(masked, torch.tensor(mask, dtype=dtype, device="cuda"), x)
    given = np.random.default_rng(v).integers(-1, v, n)
    for n_top in (20, 0):
        _check(ppas, x, given, n_top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [1500, 9001, 40000])
def test_a_row_in_batches_of_every_size(ppas, dtype, v):  # noqa: F811
    """Its tokens are the same beside any number of rows, its log probabilities within twice
    the tolerance, and, beside as many others, whatever they are, the same bits."""
    x = _logits(1400, v, seed=8, dtype=dtype)
    x[3, 7] = float("nan")
    want = None
    for n in (1, 2, 9, 20, 60, 153, 460, 700, 1400):
        rows = torch.cat([x[1000:1001], x[:n - 1]])
        a, b = _call(ppas, rows, [5] * n, 20), _call(ppas, rows, [5] * n, 20)
        assert all(np.array_equal(a[k], b[k], equal_nan=True) for k in a)
        others = _call(ppas, torch.cat([x[1000:1001], x[:n - 1].flip(1) * 3]), [5] * n, 20)
        assert all(np.array_equal(a[k][0], others[k][0]) for k in a)
        want = want or {k: t[0] for k, t in a.items()}
        assert np.array_equal(a["tok"][0], want["tok"])
        assert abs(a["lp"][0] - want["lp"]) <= 2 * (1e-5 + 2.0 ** -22 * abs(want["lp"]))
        assert abs(a["ent"][0] - want["ent"]) <= 2 * (1e-5 + 1e-5 * want["ent"])
        assert np.all(np.abs(a["top"][0] - want["top"]) <= 2 * (1e-5 + 2.0 ** -22 * np.abs(want["top"])))
