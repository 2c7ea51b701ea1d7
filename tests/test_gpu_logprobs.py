"""Log probabilities of given tokens, entropy and alternatives on the GPU, against the
float64 oracle.

Tolerance: a log probability is z - ln S.  z = x - M is rounded once (2^-24 of it, and
once more in the difference); S is a sum of positive terms, each off by at most |z| 2^-23 +
2^-22 of itself (its exponent's roundings, which weigh little where |z| is large, and
exp's), added over fewer than 128 levels of 2^-24: 8e-6 + 2^-22 + the mean of |z|
(the entropy, less than 13) times 2^-23: 1e-5 and 2^-22 of the value.  The entropy is ln S
plus a mean of |z| with the same errors: 1e-5 and 1e-5 of it."""
import numpy as np
import pytest
import torch

from oracle import logprobs as ol

pytestmark = pytest.mark.gpu

LARGEST = {torch.float32: float(np.finfo(np.float32).max), torch.bfloat16: float(torch.finfo(torch.bfloat16).max)}


@pytest.fixture(scope="module")
def ppas():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_15171_gb300 import ppas as p
    return p


def _call(ppas, x, given, n_top, **kw):
    n, v = x.shape
    got = dict(lp=torch.full((n + 1,), 7.0, device="cuda"), ent=torch.full((n + 1,), 7.0, device="cuda"),
               tok=torch.full((n + 1, n_top), -7, dtype=torch.int32, device="cuda"),
               top=torch.full((n + 1, n_top), 7.0, device="cuda"))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ppas.ppas_token_logprobs(x, x.dtype == torch.bfloat16, x.stride(0), n, v,
                             None if given is None else torch.from_numpy(np.asarray(given, np.int32)).cuda(),
                             None if given is None else got["lp"], got["ent"], n_top, got["tok"], got["top"], err, **kw)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    assert float(got["ent"][n]) == 7.0 and (n_top == 0 or int(got["tok"][n, 0]) == -7)
    return {k: t[:n].double().cpu().numpy() for k, t in got.items()}


def _near(got, want, tol):
    """equal infinities (what fp32 does not hold is one), or within tol"""
    want = np.where(want < -LARGEST[torch.float32], -np.inf, want)
    same = got == want
    with np.errstate(invalid="ignore"):
        return np.all(same | (np.abs(got - want) <= tol))


def _check(ppas, x, given, n_top):
    got = _call(ppas, x, given, n_top)
    host = x.double().cpu().numpy()
    for r in range(x.shape[0]):
        lp, ent, tok, top = ol.row(host[r], -1 if given is None else int(given[r]), n_top, LARGEST[x.dtype])
        if given is not None:
            assert _near(got["lp"][r], lp, 1e-5 + 2.0 ** -22 * abs(lp)), (r, got["lp"][r], lp)
            assert got["lp"][r] <= 0
        assert abs(got["ent"][r] - ent) <= 1e-5 + 1e-5 * ent and got["ent"][r] >= 0, (r, got["ent"][r], ent)
        assert np.array_equal(got["tok"][r], tok), r
        assert _near(got["top"][r], top, 1e-5 + 2.0 ** -22 * np.abs(top)), r


def _logits(n, v, seed, spread=3.0, dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((n, v), generator=g, device="cuda") * spread).to(dtype)


@pytest.mark.parametrize("n,v", [(1, 1), (3, 2), (2, 7), (5, 31), (4, 257), (1, 1000), (7, 4099), (1, 32003), (40, 5001),
                                 (700, 1500), (3, 152000), (1, 262144), (200, 20011)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_top", [0, 5, 32])
def test_sizes(ppas, n, v, dtype, n_top):
    x = _logits(n, v, seed=n + v, dtype=dtype)
    given = np.random.default_rng(v).integers(-1, v, size=n)
    _check(ppas, x, given, n_top)


@pytest.mark.parametrize("shift,gap", [(1, 0), (3, 5), (0, 1), (5, 11)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_alignment(ppas, shift, gap, dtype):
    n, v = 6, 3001
    base = _logits(1, n * (v + gap) + shift + 64, seed=shift, dtype=dtype)[0]
    x = base[shift:].as_strided((n, v), (v + gap, 1))
    _check(ppas, x, list(range(n)), 4)


@pytest.mark.parametrize("spread", [0.0, 1e-3, 0.3, 1.0, 10.0, 300.0, 1e5, 1e30, 3e38])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_spreads(ppas, spread, dtype):
    """From rows of one value (ties by index) to rows whose differences leave the fp32 range."""
    for n, v in ((2, 5000), (1, 70001)):
        x = (torch.rand((n, v), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") * 2 - 1) * spread
        _check(ppas, x.to(dtype), [3] * n, 20)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("v", [900, 33000])
def test_masked_infinite_and_nan_logits(ppas, dtype, v):
    x = _logits(12, v, seed=2, dtype=dtype)
    inf, nan = float("inf"), float("nan")
    x[0] = -inf                             # nothing left
    x[1] = -inf
    x[1, 700] = 2.0                         # one token left
    x[2] = -inf
    x[2, [5, 800, 6]] = torch.tensor([1.0, 1.0, 3.0], dtype=dtype, device="cuda")
    x[3, 100:600] = -inf
    x[4, 7] = inf
    x[5, [3, 899]] = inf
    x[6, 11] = nan
    x[7] = nan
    x[8, 1:] = nan
    x[9] = torch.finfo(dtype).min           # masks of the type's lowest value, everywhere
    x[10] = torch.finfo(dtype).min
    x[10, 400] = 0.5
    x[11, 0], x[11, 1] = -inf, inf
    _check(ppas, x, [5, 700, 800, 150, 7, 899, 11, 0, 0, 3, 400, 0], 8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_order_and_ties(ppas, dtype):
    """Ascending, descending and stepped rows, equal largest logits, zeros of both signs."""
    v = 40000
    up = torch.arange(v, device="cuda", dtype=torch.float32) / v * 8
    rows = [up, up.flip(0), (up * 4).floor(), torch.zeros(v, device="cuda"), torch.where(up > 4, 0.0, -0.0)]
    rows.append(torch.zeros(v, device="cuda"))
    rows[-1][torch.arange(17, v, 997, device="cuda")] = 5.0
    # the largest ones a fixed distance apart
    rows.append(-up)
    rows[-1][torch.arange(3, v, 256, device="cuda")] += 20
    rows.append(-up)
    rows[-1][torch.arange(5, v, 1024, device="cuda")] += 20
    # the second half of the row far above the first
    rows.append(torch.cat([_logits(1, v // 2, 3)[0], _logits(1, v // 2, 4)[0] + 30]))
    x = torch.stack(rows).to(dtype)
    _check(ppas, x, [v - 1] * len(rows), 32)


def test_a_sure_token(ppas):
    """Probabilities next to 1: the entropy and the largest log probability are near 0, never past it."""
    for gap in (5.0, 12.0, 17.0, 25.0, 60.0, 500.0):
        x = _logits(3, 20000, seed=6, spread=0.1)
        x[:, 77] += gap
        _check(ppas, x, [77] * 3, 2)


def test_given_token_outside_the_vocabulary(ppas):
    x = _logits(3, 500, seed=7)
    out = torch.zeros(3, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ppas.ppas_token_logprobs(x, False, 500, 3, 500, torch.tensor([4, 500, -3], dtype=torch.int32).cuda(), out,
                             d_err_flag=err)
    torch.cuda.synchronize()
    assert int(err.item()) == ppas.PPAS_DEVERR_BAD_INDEX
    assert float(out[1]) == float("-inf") and float(out[2]) == 0.0
    want = ol.row(x[0].double().cpu().numpy(), 4, 0, LARGEST[torch.float32])[0]
    assert abs(float(out[0]) - want) <= 1e-5 + 2.0 ** -22 * abs(want)


def test_rows_do_not_meet_and_repeat_bit_for_bit(ppas):
    x = _logits(300, 9001, seed=8, dtype=torch.bfloat16)
    a, b = _call(ppas, x, [5] * 300, 20), _call(ppas, x, [5] * 300, 20)
    assert all(np.array_equal(a[k], b[k]) for k in a)
    one = _call(ppas, x[250:251], [5], 20)
    assert np.array_equal(one["tok"][0], a["tok"][250]) and abs(one["lp"][0] - a["lp"][250]) < 2e-5


def test_other_stream_and_graph(ppas):
    x = _logits(20, 6000, seed=9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = _call(ppas, x, [1] * 20, 5, stream=side)
    given = torch.full((20,), 1, dtype=torch.int32, device="cuda")
    lp, ent = torch.zeros(20, device="cuda"), torch.zeros(20, device="cuda")
    tok, top = torch.zeros((20, 5), dtype=torch.int32, device="cuda"), torch.zeros((20, 5), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ppas.ppas_token_logprobs(x, False, 6000, 20, 6000, given, lp, ent, 5, tok, top)
    graph.replay()
    torch.cuda.synchronize()
    assert np.array_equal(lp.double().cpu().numpy(), a["lp"]) and np.array_equal(tok.cpu().numpy(), a["tok"])
    x.copy_(x.flip(1).contiguous())
    graph.replay()
    b = _call(ppas, x, [1] * 20, 5)
    assert np.array_equal(lp.double().cpu().numpy(), b["lp"]) and np.array_equal(tok.cpu().numpy(), b["tok"])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_past_32_bit_offsets(ppas, dtype):
    v, stride = 3000, (1 << 30) + 5
    x = torch.empty(3 * stride, dtype=dtype, device="cuda").as_strided((3, v), (stride, 1))
    x.copy_(_logits(3, v, seed=11, dtype=dtype))
    _check(ppas, x, [7, 2999, 0], 9)


def test_long_lists_of_few_lanes(ppas):
    """More logits at the bound than a warp's list holds: all of them in one lane's, or one warp's, places."""
    v = 30000
    for first, step, count in ((64, 1024 * 8, 40), (0, 1, 400), (2048, 4, 300), (5, 32, 200)):
        for dtype in (torch.float32, torch.bfloat16):
            x = _logits(2, v, seed=12, spread=0.5, dtype=dtype)
            at = (first + step * torch.arange(count, device="cuda")) % v
            x[:, at] = (20 + torch.randn(2, count, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))).to(dtype)
            _check(ppas, x, [int(at[0]), int(at[-1])], 32)


def test_two_streams_at_once(ppas):
    xs = [_logits(40, 20000, seed=13), _logits(300, 9000, seed=14)]
    streams = [torch.cuda.Stream() for _ in xs]
    alone = [_call(ppas, x, [3] * x.shape[0], 10) for x in xs]
    outs = []
    for x in xs:
        n = x.shape[0]
        outs.append((torch.full((n,), 3, dtype=torch.int32, device="cuda"), torch.empty(n, device="cuda"),
                     torch.empty(n, device="cuda"), torch.empty((n, 10), dtype=torch.int32, device="cuda"),
                     torch.empty((n, 10), device="cuda")))
    torch.cuda.synchronize()
    for _ in range(20):
        for x, o, s in zip(xs, outs, streams):
            ppas.ppas_token_logprobs(x, False, x.stride(0), x.shape[0], x.shape[1], o[0], o[1], o[2], 10, o[3], o[4], None, s)
    torch.cuda.synchronize()
    for a, o in zip(alone, outs):
        for k, t in zip(("lp", "ent", "tok", "top"), o[1:]):
            assert np.array_equal(a[k], t.double().cpu().numpy())


# rows that are many and short: CTAs of 64 and of 128 threads
@pytest.mark.parametrize("n,v", [(153, 1), (160, 7), (200, 33), (310, 2047), (153, 2048), (700, 2049), (1300, 2050), (1300, 8192),
                                 (700, 8193), (700, 16384), (1300, 20011)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_top", [0, 1, 32])
def test_many_short_rows(ppas, n, v, dtype, n_top):
    shift = n_top % 5
    x = _logits(n, v + 3 * shift, seed=n + v, dtype=dtype)[:, shift:shift + v]
    given = np.random.default_rng(v).integers(-1, v, n)
    _check(ppas, x, given, n_top)


@pytest.mark.parametrize("n,v", [(180, 900), (1300, 5000), (700, 9000), (1300, 17000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_short_rows_of_every_kind(ppas, n, v, dtype):
    x = _logits(n, v, seed=v, dtype=torch.float32)
    kinds = 12
    at = torch.arange(n, device="cuda") % kinds
    ramp = torch.linspace(-40, 40, v, device="cuda")
    x[at == 1] = -float("inf")
    x[at == 2] = 1.5
    x[at == 3] = ramp
    x[at == 4] = ramp.flip(0)
    x[at == 5] = (x[at == 5] * 2).round()          # many equal ones
    x[at == 6] = x[at == 6] * 1e37
    x[at == 7] = torch.where(x[at == 7] > 0, x[at == 7], -float("inf"))
    x[at == 8] = torch.where(x[at == 8] > 0, x[at == 8], float("nan"))
    x[at == 9, v // 2] = float("inf")
    x[at == 10, :-1] = -float("inf")               # a sure token
    x[at == 11] = x[at == 11] * 1e-3 - 1e30
    x = x.to(dtype)
    given = np.random.default_rng(v).integers(-1, v, n)
    _check(ppas, x, given, 20)
    _check(ppas, x, given, 0)
