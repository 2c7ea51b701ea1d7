"""Low-rank adapters of many requests on the GPU, every element against the float64
oracle (``oracle.adapter.bound`` says how far off a result may be, and why)."""
import numpy as np
import pytest
import torch

from oracle import adapter as oad

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ppas():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_15171_gb300 import ppas as p
    return p


def _normal(shape, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


class Call:
    def __init__(self, lens, ids, hidden, slices, rank, n_adapters=None, seed=0, gap=0, scales=True):
        self.lens, self.ids = np.array(lens, np.int32), np.array(ids, np.int32)
        self.n = int(max(ids)) + 1 if n_adapters is None else n_adapters
        self.n = max(self.n, 1)
        t, self.hidden, self.rank = int(self.lens.sum()), hidden, rank
        self.slices, cols = np.array(slices, np.int32), int(sum(slices))
        self.T, self.cols = t, cols
        self.x = _normal((t + 3, hidden + gap), seed + 1)[:t, :hidden]
        self.y = _normal((t + 3, cols + gap), seed + 2)[:t, :cols]
        self.full = torch.full((t + 3, cols + gap), 9.0, dtype=torch.bfloat16, device="cuda")
        self.out = self.full[:t, :cols]
        self.a = _normal((self.n, len(slices) * rank, hidden), seed + 3, hidden ** -0.5)
        self.b = _normal((self.n, cols, rank), seed + 4, rank ** -0.5)
        self.scales = torch.from_numpy(np.random.default_rng(seed).normal(size=self.n).astype(np.float32)).cuda() \
            if scales else None
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def args(self, **kw):
        a = dict(x=self.x, x_stride=self.x.stride(0), y=self.y, y_stride=self.y.stride(0), out=self.out,
                 out_stride=self.out.stride(0), q_lens=self.lens, adapters=self.ids, a=self.a, b=self.b,
                 d_scales=self.scales, n_adapters=self.n, hidden=self.hidden, slice_cols=self.slices, rank=self.rank,
                 d_err_flag=self.err)
        a.update(kw)
        return a

    def host(self):
        f = lambda v: None if v is None else v.double().cpu().numpy()  # noqa: E731
        return (f(self.x), f(self.y), self.lens, self.ids, f(self.a), f(self.b), f(self.scales), self.slices, self.rank)

    def check(self, host=None):
        torch.cuda.synchronize()
        assert int(self.err.item()) == 0
        h = self.host() if host is None else host
        off = np.abs(self.out.double().cpu().numpy() - oad.adapter_add(*h)) - oad.bound(*h)
        assert np.all(off <= 0), off.max()
        # rows behind the last sequence and columns past the last slice as they were
        assert bool((self.full[self.T:] == 9.0).all()) and bool((self.full[:, self.cols:] == 9.0).all())
        rows = torch.from_numpy(np.repeat(self.ids, self.lens) < 0).cuda()
        assert torch.equal(self.out[rows], self.y[rows])


@pytest.mark.parametrize("lens,ids", [
    ([1], [0]), ([1], [-1]), ([2], [1]), ([1] * 5, [0, 1, 0, -1, 1]), ([1] * 64, list(range(64))),
    ([1] * 40, [0] * 40), ([1] * 70, [0, 3] * 35), ([1, 1, 15, 16, 17, 1], [2, 2, 1, 2, -1, 0]),
    ([127], [0]), ([128], [0]), ([129], [0]), ([300, 1, 5, 200], [1, 1, 0, 2]), ([64, 65, 63], [0, 0, 1]),
    ([1, 1, 1, 513, 255, 700], [4, 0, -1, 2, -1, 4]), ([33, 40, 47, 48, 49, 95], [0, 1, 0, 1, 2, 0])])
@pytest.mark.parametrize("hidden,slices,rank", [(2048, [2048, 256, 256], 16), (512, [384], 8), (256, [72, 200, 8], 24)])
def test_batches(ppas, lens, ids, hidden, slices, rank):
    c = Call(lens, ids, hidden, slices, rank, seed=len(lens))
    ppas.ppas_adapter_add(**c.args())
    c.check()


@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 64, 104, 128])
@pytest.mark.parametrize("slices", [[256], [136, 40], [320, 64, 64], [8, 8, 16, 24]])
def test_ranks_and_slices(ppas, rank, slices):
    for lens, ids in (([1, 1, 1], [0, 1, 0]), ([1, 150, 260], [1, 0, 1])):
        c = Call(lens, ids, 320, slices, rank, seed=rank)
        ppas.ppas_adapter_add(**c.args())
        c.check()


@pytest.mark.parametrize("hidden", [8, 16, 56, 64, 72, 136, 1000, 4096, 11008])
@pytest.mark.parametrize("cols", [8, 64, 264])
def test_hidden_sizes(ppas, hidden, cols):
    for lens, ids in (([1, 1], [0, 1]), ([3, 140], [1, 0])):
        c = Call(lens, ids, hidden, [cols], 16, seed=hidden + cols, gap=8)
        ppas.ppas_adapter_add(**c.args())
        c.check()


def test_strides_in_place_and_no_scales(ppas):
    for lens, ids in (([1, 1, 20], [0, -1, 1]), ([200, 130, 1], [1, -1, 0])):
        c = Call(lens, ids, 256, [128, 64], 16, seed=5, gap=24, scales=False)
        host = c.host()
        c.full[:c.T, :c.cols] = c.y
        c.y = c.out
        ppas.ppas_adapter_add(**c.args(y=c.out, y_stride=c.out.stride(0)))
        c.check(host)


def test_many_adapters_past_32_bit_offsets(ppas):
    """Weights beyond 2^31 elements."""
    n, hidden, rank = 2100, 16384, 64
    c = Call([1, 1, 140], [2099, 2050, 2098], hidden, [64], rank, n_adapters=1, seed=6)
    c.n = n
    c.a = torch.zeros((n, rank, hidden), dtype=torch.bfloat16, device="cuda")
    c.b = torch.zeros((n, 64, rank), dtype=torch.bfloat16, device="cuda")
    c.scales = torch.ones(n, device="cuda")
    for i, k in enumerate((2099, 2050, 2098)):
        c.a[k] = _normal((rank, hidden), 50 + i, hidden ** -0.5)
        c.b[k] = _normal((64, rank), 60 + i, rank ** -0.5)
    ppas.ppas_adapter_add(**c.args())
    used = [2099, 2050, 2098]
    f = lambda v: v.double().cpu().numpy()  # noqa: E731
    c.check((f(c.x), f(c.y), c.lens, np.array([0, 1, 2]), f(c.a[used]), f(c.b[used]), np.ones(3), c.slices, rank))


def test_rows_do_not_meet(ppas):
    """NaN and infinities of one row, and of adapters that it does not have, stay away from the others."""
    for lens, ids in (([1] * 12, [0, 1] * 6), ([130, 1, 129], [0, 1, 2])):
        c = Call(lens, ids, 256, [192], 16, n_adapters=4, seed=7)
        clean = Call(lens, ids, 256, [192], 16, n_adapters=4, seed=7)
        c.x[3] = float("nan")
        c.x[9, 5] = float("inf")
        c.a[3], c.b[3] = float("nan"), float("nan")
        for v in (c, clean):
            ppas.ppas_adapter_add(**v.args())
        torch.cuda.synchronize()
        same = torch.ones(c.T, dtype=torch.bool, device="cuda")
        same[3] = same[9] = False
        assert torch.equal(c.out[same], clean.out[same])
        assert bool(c.out[3].isnan().all())


def test_repeats_bit_for_bit(ppas):
    lens, ids = [1] * 30 + [700, 90], [i % 7 for i in range(30)] + [3, 4]
    c = Call(lens, ids, 2048, [512, 128, 128], 32, seed=8)
    ppas.ppas_adapter_add(**c.args())
    first = c.full.clone()
    for _ in range(3):
        c.out.fill_(1.0)
        ppas.ppas_adapter_add(**c.args())
        assert torch.equal(c.full, first)


def test_many_sequences(ppas):
    """More units and rows than one launch's tables hold."""
    rng = np.random.default_rng(0)
    lens = [1] * 5000 + [int(x) for x in rng.integers(1, 40, size=700)]
    ids = [int(x) for x in rng.integers(-1, 900, size=5700)]
    c = Call(lens, ids, 64, [40], 8, seed=9)
    ppas.ppas_adapter_add(**c.args())
    c.check()


def test_other_stream_and_graph(ppas):
    for lens, ids in (([1] * 9, [0, 1, 2] * 3), ([140, 1, 300], [0, 1, -1])):
        c = Call(lens, ids, 256, [128], 16, seed=10)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        ppas.ppas_adapter_add(**c.args(stream=side))
        side.synchronize()
        c.check()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ppas.ppas_adapter_add(**c.args())
        c.x.mul_(-0.5)
        c.y.mul_(2.0)
        c.out.fill_(0.0)
        graph.replay()
        c.check()


# ---- runs of more than 512 rows, which are done in tiles of 128 (short runs beside them in units)
@pytest.mark.parametrize("rank", [8, 16, 24, 32, 40, 64, 72, 104, 128])
@pytest.mark.parametrize("slices", [[256], [136, 40], [320, 64, 64], [8, 8, 16, 24]])
def test_tiles_ranks_and_slices(ppas, rank, slices):
    for lens, ids in (([1, 150, 470], [1, 0, 1]), ([513], [0])):
        c = Call(lens, ids, 320, slices, rank, seed=rank)
        ppas.ppas_adapter_add(**c.args())
        c.check()


@pytest.mark.parametrize("hidden", [8, 56, 64, 72, 136, 200, 264, 1000, 4096])
@pytest.mark.parametrize("cols", [8, 72, 264, 1032])
def test_tiles_hidden_sizes(ppas, hidden, cols):
    """From one block of K, and a cluster of one CTA, to clusters of eight."""
    c = Call([2, 140, 513], [0, 1, 0], hidden, [cols], 16, seed=hidden + cols, gap=8)
    ppas.ppas_adapter_add(**c.args())
    c.check()


@pytest.mark.parametrize("tiles", [5, 9, 15, 16, 23, 24, 28, 36, 37, 50, 76, 77, 100, 153])
def test_tiles_counts(ppas, tiles):
    """Clusters of every size, to single CTAs in more than one round."""
    rows = [128 * (tiles - 3) - 5, 48, 101]  # 3 + (tiles - 3) tiles of three runs
    c = Call([1] + rows, [0, 1, 2, 0], 520, [136, 64], 16, seed=tiles)
    ppas.ppas_adapter_add(**c.args())
    c.check()


def test_tiles_wide_inner_sums(ppas):
    """384 inner sums, of 256 and 128 in two products; rows of the last tile few."""
    for rows in (514, 900, 10000):
        c = Call([rows], [1], 512, [128, 64, 40], 128, seed=rows)
        ppas.ppas_adapter_add(**c.args())
        c.check()


def test_tiles_strides_in_place_and_no_scales(ppas):
    for lens, ids in (([600, 130, 1], [1, -1, 0]), ([1, 512, 200], [0, 0, 1])):
        c = Call(lens, ids, 256, [128, 72], 16, seed=5, gap=24, scales=False)
        host = c.host()
        c.full[:c.T, :c.cols] = c.y
        c.y = c.out
        ppas.ppas_adapter_add(**c.args(y=c.out, y_stride=c.out.stride(0)))
        c.check(host)


def test_tiles_rows_do_not_meet(ppas):
    """NaN and infinities of one row, and of the adapters before and behind, stay away from the others."""
    for rank in (8, 16, 40):
        for slices in ([200], [72, 136]):
            c = Call([700, 2, 100], [1, 2, 1], 328, slices, rank, n_adapters=4, seed=7)
            clean = Call([700, 2, 100], [1, 2, 1], 328, slices, rank, n_adapters=4, seed=7)
            c.x[3] = float("nan")
            c.x[690, 5] = float("inf")
            c.y[128, 9] = float("nan")
            for k in (0, 3):
                c.a[k], c.b[k] = float("nan"), float("nan")
            for v in (c, clean):
                ppas.ppas_adapter_add(**v.args())
            torch.cuda.synchronize()
            same = torch.ones_like(c.out, dtype=torch.bool)
            same[3] = same[690] = False
            same[128, 9] = False
            assert torch.equal(c.out[same], clean.out[same])
            assert bool(c.out[3].isnan().all()) and bool(c.out[128, 9].isnan())


def test_tiles_past_32_bit_offsets(ppas):
    """Rows of x and out further than 2^31 elements apart, and weights behind 2^31."""
    t, stride = 600, 1 << 23
    c = Call([t], [0], 128, [64], 16, seed=12)
    x = torch.zeros((t, stride), dtype=torch.bfloat16, device="cuda")
    x[:, :128] = c.x
    n = 1 << 14
    a = torch.zeros((n, 16, 16384), dtype=torch.bfloat16, device="cuda")
    b = torch.zeros((n, 64, 16), dtype=torch.bfloat16, device="cuda")
    out = torch.empty((t, stride), dtype=torch.bfloat16, device="cuda")
    a = a.view(n * 128, 16, 128)
    c.lens, c.ids = np.array([t], np.int32), np.array([n - 1], np.int32)
    a[n - 1], b[n - 1] = c.a[0], c.b[0]
    scales = torch.ones(n, device="cuda")
    scales[n - 1] = c.scales[0]
    ppas.ppas_adapter_add(**c.args(x=x, x_stride=stride, out=out, out_stride=stride, a=a, b=b, d_scales=scales,
                                   n_adapters=n))
    c.out.copy_(out[:, :64])
    c.ids = np.array([0], np.int32)
    c.check()
    # the last adapter's weights lie behind 2^31 elements
    big = torch.zeros((n, 16, 16384), dtype=torch.bfloat16, device="cuda")
    x2 = _normal((t, 16384), 3)
    d = Call([t], [0], 16384, [64], 16, seed=13)
    d.x = x2
    big[n - 1], b[n - 1] = d.a[0], d.b[0]
    scales[n - 1] = d.scales[0]
    ppas.ppas_adapter_add(**d.args(a=big, b=b, d_scales=scales, n_adapters=n, adapters=[n - 1]))
    d.check()


def test_calls_behind_one_another(ppas):
    """Each call reads what the one before wrote, tiles and units in all of them, and a graph of them."""
    lens, ids = [1, 600, 1, 1, 300, 20], [1, 0, -1, 0, 2, 1]
    layers = [Call(lens, ids, 256, [256], 16, n_adapters=3, seed=20 + i) for i in range(6)]

    def chain(wait):
        x = layers[0].x
        for c in layers:
            ppas.ppas_adapter_add(**c.args(x=x, x_stride=x.stride(0)))
            if wait:
                torch.cuda.synchronize()
            x = c.out
    chain(True)
    want = [c.full.clone() for c in layers]
    for _ in range(5):
        for c in layers:
            c.out.fill_(float("nan"))
        chain(False)
        torch.cuda.synchronize()
        assert all(torch.equal(c.full, w) for c, w in zip(layers, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(False)
    for _ in range(5):
        for c in layers:
            c.out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(c.full, w) for c, w in zip(layers, want))


def test_two_streams_at_once(ppas):
    """Calls of two streams, and of two captured graphs, share nothing."""
    a = Call([1, 700, 1, 30], [0, 1, 1, 0], 512, [192, 64], 16, seed=30)
    b = Call([900, 1, 1], [1, 0, 1], 512, [192, 64], 16, seed=31)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        for c, s in zip((a, b), streams):
            ppas.ppas_adapter_add(**c.args(stream=s))
    torch.cuda.synchronize()
    a.check()
    b.check()
    graphs = []
    for c in (a, b):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            ppas.ppas_adapter_add(**c.args())
        c.out.fill_(0.0)
    torch.cuda.synchronize()
    for _ in range(10):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    a.check()
    b.check()


# tiles of 64 rows: few enough rows that all of them run at a time, inner sums that make up for it
@pytest.mark.parametrize("rank", [8, 16, 40, 64, 128])
@pytest.mark.parametrize("hidden,slices", [(2048, [1024, 256, 256]), (1000, [264, 72]), (520, [200])])
def test_half_tiles(ppas, rank, hidden, slices):
    for lens, ids in (([300, 100, 77, 129, 1], [0, 1, 0, 2, -1]), ([64, 65, 63, 200, 191], [0, 1, 2, 0, 3]), ([768], [0])):
        c = Call(lens, ids, hidden, slices, rank, seed=rank)
        ppas.ppas_adapter_add(**c.args())
        c.check()


def test_half_tiles_in_place_and_strides(ppas):
    c = Call([400, 333, 48], [0, 1, 0], 2048, [1024, 264, 256], 64, gap=24, seed=5, scales=False)
    h = c.host()
    c.out.copy_(c.y)
    ppas.ppas_adapter_add(**c.args(y=c.out, y_stride=c.out.stride(0)))
    c.check(h)


# few rows of wide inner sums or many columns: a row's cluster has 16 CTAs
@pytest.mark.parametrize("hidden,slices,rank", [(4096, [64, 8, 24], 64), (4104, [2048, 2048, 2056], 16), (11008, [264], 40),
                                                (2048, [4096, 1000], 128), (2056, [8] * 4, 128)])
@pytest.mark.parametrize("ids", [[0], [-1], [0, 0], [0, 1, 0, 2], [0] * 4, [4, -1, 2, 3, 1], list(range(7)), list(range(12)),
                                 [0] * 9])
def test_long_rows_few_at_a_time(ppas, hidden, slices, rank, ids):
    c = Call([1] * len(ids), ids, hidden, slices, rank, seed=len(ids))
    ppas.ppas_adapter_add(**c.args())
    c.check()
