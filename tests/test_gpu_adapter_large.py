"""Adapter steps of so many rows that tiles need the large table, several launches, or units
behind them more than one: every element against the float64 oracle, and a chain of dependent
calls without a host wait against the same chain with waits."""
import numpy as np
import pytest
import torch

from test_gpu_adapter import Call, ppas  # noqa: F401

pytestmark = pytest.mark.gpu


def _singles(n, ids, seed):
    """n sequences of one row, one in ten without an adapter, else of adapters in a random order."""
    rng = np.random.default_rng(seed)
    which = rng.integers(1, ids, size=n)
    which[rng.random(n) < 0.1] = -1
    return [1] * n, [int(x) for x in which]


def _steps():
    some = _singles(60, 9, 1)
    many = _singles(5600, 1500, 2)
    return {
        # (2 KB of parameters hold 160 tiles, 32 KB 2600)
        "161 tiles": ([128 * 160 + 5], [0]),
        "200 tiles beside units": (some[0] + [128 * 199 + 40, 47], some[1] + [0, 3]),
        "two launches of tiles": ([128 * 2600 + 1], [0]),
        "two launches of tiles, beside units": (some[0] + [128 * 2700 + 77, 300, 15], some[1] + [0, 2, 4]),
        # (a launch of units holds 1024, and 3584 listed rows)
        "three launches of units beside tiles": (many[0] + [600], many[1] + [0]),
        "units before and behind tiles": (many[0][:3000] + [700, 20, 513] + many[0][3000:], many[1][:3000] + [0, 5, 0] + many[1][3000:]),
        "units beside many tiles": (many[0] + [128 * 170], many[1] + [0]),
    }


@pytest.mark.parametrize("name", list(_steps()))
def test_rows(ppas, name):  # noqa: F811
    lens, ids = _steps()[name]
    c = Call(lens, ids, 64, [40], 8, seed=len(lens))
    ppas.ppas_adapter_add(**c.args())
    c.check()


@pytest.mark.parametrize("name", list(_steps()))
def test_rows_in_place(ppas, name):  # noqa: F811
    lens, ids = _steps()[name]
    c = Call(lens, ids, 64, [24, 16], 8, seed=len(lens), gap=8, scales=False)
    host = c.host()
    c.full[:c.T, :c.cols] = c.y
    c.y = c.out
    ppas.ppas_adapter_add(**c.args(y=c.out, y_stride=c.out.stride(0)))
    c.check(host)


@pytest.mark.parametrize("name", list(_steps()))
def test_calls_behind_one_another(ppas, name):  # noqa: F811
    """Each call reads what the one before wrote, the last one in place over its own input's source."""
    lens, ids = _steps()[name]
    layers = [Call(lens, ids, 64, [64], 8, seed=20 + i) for i in range(3)]

    def chain(wait):
        x = layers[0].x
        for i, c in enumerate(layers):
            ppas.ppas_adapter_add(**c.args(x=x, x_stride=x.stride(0)))
            if wait:
                torch.cuda.synchronize()
            x = c.out
        # in place, over what the second call has read
        c = layers[0]
        ppas.ppas_adapter_add(**c.args(x=x, x_stride=x.stride(0), y=c.out, y_stride=c.out.stride(0)))
        torch.cuda.synchronize()
    chain(True)
    want = [c.full.clone() for c in layers]
    for _ in range(3):
        for c in layers:
            c.out.fill_(float("nan"))
        torch.cuda.synchronize()
        chain(False)
        assert all(torch.equal(c.full, w) for c, w in zip(layers, want))
    assert all(int(c.err.item()) == 0 for c in layers)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x = layers[0].x
        for c in layers:
            ppas.ppas_adapter_add(**c.args(x=x, x_stride=x.stride(0)))
            x = c.out
    for c in layers:
        c.out.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(c.full, w) for c, w in zip(layers[1:], want[1:]))
