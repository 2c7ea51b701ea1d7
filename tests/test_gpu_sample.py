"""Sampling on the GPU: tokens and log-probabilities against the float64 oracle
(at the edges of rules, types, sizes and alignments), token for token against
the whole-number definition, the same row in any batch, and the frequencies of
many draws.

Tolerance: z, exp and the product with 2^40 are fp32 (z off by up to 2 units of
2^-24 of |z| <= 28, so a weight by 28 * 2^-23 + 2^-23 of itself) and a weight is
cut by less than 2^-40, of a sum that is at least 1: running sums are good to
4e-6 + vocab 2^-40, taken as 1e-5."""
import math

import numpy as np
import pytest
import torch

from oracle import sampling as so

pytestmark = pytest.mark.gpu
TOL = 1e-5


@pytest.fixture(scope="module")
def ppas():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_15171_gb300 import ppas as p
    return p


def _call(ppas, x, temperature=None, top_k=None, top_p=None, min_p=None, u=None, logprobs=True, **kw):
    n, v = x.shape

    def dev(a, t):
        return None if a is None else torch.as_tensor(np.broadcast_to(np.asarray(a), (n,)).copy(), dtype=t).cuda()
    tokens = torch.full((n + 1,), -7, dtype=torch.int32, device="cuda")
    lp = torch.full((n + 1,), 9.0, dtype=torch.float32, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    args = [dev(temperature, torch.float32), dev(top_k, torch.int32), dev(top_p, torch.float32),
            dev(min_p, torch.float32), dev(0.5 if u is None else u, torch.float32)]
    torch.cuda.synchronize()
    ppas.ppas_sample_tokens(x, x.dtype == torch.bfloat16, x.stride(0), n, v, *args, tokens,
                            lp if logprobs else None, err, **kw)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    assert int(tokens[n]) == -7 and float(lp[n]) == 9.0
    return tokens[:n].cpu().numpy(), lp[:n].cpu().numpy()


def _logits(n, v, seed, spread=3.0, bf16=False):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((n, v), generator=g, device="cuda") * spread
    return x.to(torch.bfloat16) if bf16 else x


RULES = [(1.0, 0, 1.0, 0.0), (0.8, 0, 0.95, 0.0), (0.7, 50, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.05),
         (0.6, 40, 0.9, 0.02), (1.3, 1000, 0.98, 0.0), (2.0, 1, 0.9, 0.0), (1.0, 3, 0.01, 0.5)]


def _check(x, rules, u, tokens, lp, rows=None):
    xs = x.float().cpu().numpy()
    f32 = np.float32
    for r in range(len(xs)) if rows is None else rows:
        t, k, p, m = rules[r]
        assert so.accepts(tokens[r], lp[r], xs[r], float(f32(t)), k, float(f32(p)), float(f32(m)), float(f32(u[r])),
                          TOL), (r, rules[r], u[r], tokens[r], lp[r], so.sample(xs[r], t, k, p, m, u[r]))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("v", [1, 2, 7, 31, 100, 1000, 1023, 4097, 8193, 32003, 128000])
def test_rules_over_vocabularies(ppas, v, bf16):
    n = 36
    x = _logits(n, v, v, 3.0, bf16)
    rng = np.random.default_rng(v)
    rules = [RULES[r % len(RULES)] for r in range(n)]
    u = rng.random(n).astype(np.float32)
    u[:9], u[9:18] = 0.0, 1 - 2.0 ** -24
    tokens, lp = _call(ppas, x, *zip(*rules), u)
    _check(x, rules, u, tokens, lp)


@pytest.mark.parametrize("n,v", [(1, 262144), (1, 152000), (3, 152000), (19, 200003), (40, 152000), (200, 152000),
                                 (300, 5000), (1000, 300)])
def test_batches(ppas, n, v):
    x = _logits(n, v, n + v, 2.0)
    rng = np.random.default_rng(n)
    rules = [RULES[(r * 5) % len(RULES)] for r in range(n)]
    u = rng.random(n).astype(np.float32)
    tokens, lp = _call(ppas, x, *zip(*rules), u)
    _check(x, rules, u, tokens, lp, rows=range(0, n, max(1, n // 40)))


def _whole_numbers(x, t, k, p, m, u):
    """The definition in whole numbers on the device (fp32 exp, 64-bit sums), one row."""
    x = x.float() + 0.0
    x = torch.where(torch.isnan(x), -math.inf, x)
    top, v = x.max(), x.numel()
    if t <= 0:
        return int(torch.argmax((x == top).to(torch.int32)))
    z = torch.where(x == top, 0.0, (x - top) * (1.0 / torch.tensor(t, dtype=torch.float32, device="cuda")))
    w = torch.where(x == -math.inf, 0.0, torch.exp(z))
    w = (w.double() * 2.0 ** 40).to(torch.int64)
    order = torch.sort(x, descending=True, stable=True).indices
    cum = torch.cumsum(w[order], 0)
    n = k if 0 < k < v else v
    if p < 1:
        n = min(n, 1 + int((cum < math.ceil(float(np.float32(p)) * float(cum[n - 1]))).sum()))
    if m > 0:
        n = max(1, min(n, int((z >= torch.log(torch.tensor(m, dtype=torch.float32, device="cuda"))).sum())))
    s = int(cum[n - 1])
    at = min(int(float(np.float32(u)) * float(s)), s - 1)
    return int(order[int((cum <= at).sum())])


@pytest.mark.parametrize("spread,bf16,v", [(3.0, False, 32003), (0.02, False, 32003), (3.0, True, 32003),
                                           (0.3, True, 100000), (8.0, False, 152000)])
def test_token_for_token(ppas, spread, bf16, v):
    n = 45
    x = _logits(n, v, 77, spread, bf16)
    rules = [RULES[r % len(RULES)] for r in range(n)]
    u = np.random.default_rng(5).random(n).astype(np.float32)
    tokens, _ = _call(ppas, x, *zip(*rules), u)
    for r in range(n):
        assert tokens[r] == _whole_numbers(x[r], *rules[r], u[r]), (r, rules[r])


@pytest.mark.parametrize("v", [5, 3000, 70000, 262144])
def test_equal_logits(ppas, v):
    """A row of one value: every cut and the draw go by the index, up to a whole vocabulary of ties."""
    x = torch.full((6, v), -2.5, device="cuda")
    k = [0, v // 2 + 1, 0, 3, 0, 0]
    p = [1.0, 1.0, 0.25, 1.0, 0.5, 1.0]
    u = np.array([0.999, 0.999, 0.999, 0.999, 0.0, 0.3], np.float32)
    tokens, lp = _call(ppas, x, 0.7, k, p, 0.0, u)
    for r in range(6):
        n = k[r] if 0 < k[r] < v else v
        n = math.ceil(p[r] * n) if p[r] < 1 else n
        assert tokens[r] == min(int(float(u[r]) * n), n - 1), r
        assert abs(lp[r] + math.log(n)) < 1e-6 * max(1, math.log(n))


def test_few_distinct_values(ppas):
    """Thousands of ties at each value: bins that are divided by value, then by index."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randint(0, 7, (30, 90000), generator=g, device="cuda").float() * 0.5
    rules = [(1.0, 0, 1.0, 0.0), (1.0, 20000, 1.0, 0.0), (0.5, 0, 0.9, 0.0), (1.0, 40000, 0.5, 0.0),
             (3.0, 0, 0.3, 0.4)] * 6
    u = np.random.default_rng(4).random(30).astype(np.float32)
    for y in (x, x.to(torch.bfloat16)):
        tokens, lp = _call(ppas, y, *zip(*rules), u)
        for r in range(30):
            assert tokens[r] == _whole_numbers(y[r], *rules[r], u[r]), r
        _check(y, rules, u, tokens, lp)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n", [1, 2, 31, 127, 128, 129, 300, 511, 512, 513, 1000])
def test_tokens_of_one_value(ppas, n, bf16):
    """n ties, some larger and many smaller logits: top-k, top-p and the draw all end inside the ties."""
    v, reps = 20000, 8
    g = np.random.default_rng(n)
    x = np.full((reps, v), -math.inf, np.float32)
    for r in range(reps):
        at = g.permutation(v)
        x[r, at[:n]] = 1.0
        x[r, at[n:n + 5]] = [1.25, 1.5, 1.5, 2.0, 3.0]
        x[r, at[n + 5:]] = -9.0 - g.integers(0, 64, v - n - 5) / 8
    x = torch.from_numpy(x).cuda()
    x = x.to(torch.bfloat16) if bf16 else x
    rules = [(1.0, 0, 1.0, 0.0), (0.8, n // 2 + 6, 1.0, 0.0), (1.0, 0, 0.9, 0.0), (1.0, n // 2 + 6, 0.95, 0.1)] * 2
    u = np.array([0.5, 0.9, 0.97, 0.8, 0.9999, 0.99999, 0.999, 0.98], np.float32)
    tokens, lp = _call(ppas, x, *zip(*rules), u)
    for r in range(reps):
        assert tokens[r] == _whole_numbers(x[r], *rules[r], u[r]), (r, rules[r])
    _check(x, rules, u, tokens, lp)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("stride", [90000, 90003])
def test_few_large_logits_in_long_rows(ppas, stride, bf16):
    """Rows too many and long for shared memory, of nothing, NaN or far smaller logits but for a handful of
    tokens at the start, the end and between: the passes over most of a row have nothing to find."""
    n, v = 320, 90000
    x = torch.full((n, stride), -math.inf, device="cuda", dtype=torch.bfloat16 if bf16 else torch.float32)
    g = np.random.default_rng(6)
    for r in range(n):
        if r % 3 == 1:
            x[r] = math.nan
        elif r % 3 == 2:
            x[r] = -20.0
        where = g.choice([0, 1, 2, 3, 7, 8191, 8192, 8193, 44999, 45000, 45001, 65535, v - 9, v - 2, v - 1], 6,
                         replace=False)
        x[r, torch.from_numpy(where).cuda()] = torch.from_numpy(g.integers(-8, 9, 6) / 4).to(x)
    rules = [RULES[r % len(RULES)] for r in range(n)]
    u = g.random(n).astype(np.float32)
    tokens, _ = _call(ppas, x[:, :v], *zip(*rules), u)
    for r in range(n):
        assert tokens[r] == _whole_numbers(x[r, :v], *rules[r], u[r]), (r, rules[r])


def test_special_values(ppas):
    inf, nan = math.inf, math.nan
    low32, low16 = -3.4028234663852886e38, -3.3895313892515355e38
    rows = [
        [-inf] * 9, [nan] * 9, [nan, -inf, 2.0, -inf, nan, -inf, -inf, -inf, -inf],  # nothing, nothing, one token
        [inf, 1.0, inf, -inf, nan, 3.0, 0.0, 0.0, inf],  # shared by the three infinities
        [low32] * 9, [low32, 1.0, low32, low32, 1.0, low32, low32, low32, low32], [low16] * 8 + [low32],
        [0.0, -0.0, 0.0, -0.0, -0.0, 0.0, -0.0, 0.0, -0.0],  # one value: the lowest index first
        [3.0e38, -3.0e38, 3.0e38, 0.0, 1.0, 2.0, 3.0, 4.0, 5.0], [1e-45, 0.0, -1e-45] * 3,
    ]
    x = torch.tensor(rows, device="cuda")
    n = len(rows)
    for t in (1.0, 0.0, 1e-6, 1e6, 0.3):
        for k, p, m in ((0, 1.0, 0.0), (2, 1.0, 0.0), (0, 0.6, 0.0), (0, 1.0, 0.5)):
            for u in (0.0, 0.5, 0.99):
                tokens, lp = _call(ppas, x, t, k, p, m, u)
                assert list(tokens[:2]) == [-1, -1] and np.all(lp[:2] == -inf) and tokens[2] == 2 and lp[2] == 0
                assert tokens[3] in (0, 2, 8)
                _check(x, [(t, k, p, m)] * n, [u] * n, tokens, lp)
    # ties of zeros of both signs go by index
    tokens, _ = _call(ppas, x[7:8], 1.0, 0, 1.0, 0.0, 0.5)
    assert tokens[0] == 4


def test_outliers_and_temperatures(ppas):
    """A few values far off the rest spread the bins thin; extreme temperatures."""
    x = _logits(8, 50000, 9, 1e-3)
    x[:, 7] = -1e30
    x[:4, 11] = 50.0
    x[2, 100:40000] = -math.inf
    for t in (1e-30, 1e-3, 1.0, 1e3, 1e30):
        for k, p in ((0, 1.0), (700, 0.9)):
            rules = [(t, k, p, 0.0)] * 8
            u = np.linspace(0, 0.999, 8).astype(np.float32)
            tokens, lp = _call(ppas, x, t, k, p, 0.0, u)
            for r in range(8):
                assert tokens[r] == _whole_numbers(x[r], t, k, p, 0.0, u[r]), (t, k, r)
            if 1e-3 <= t <= 1e3:
                _check(x, rules, u, tokens, lp)


def test_rule_edges(ppas):
    """Rules that leave one token or all, and numbers outside their ranges."""
    x = _logits(1, 5000, 4)
    first = int(x[0].argmax())
    for kw in (dict(top_k=1), dict(top_p=0.0), dict(top_p=-1.0), dict(top_p=1e-9), dict(min_p=1.0), dict(min_p=7.0),
               dict(temperature=0.0), dict(temperature=-2.0), dict(temperature=math.nan), dict(temperature=1e-38)):
        tokens, lp = _call(ppas, x, u=0.9999, **kw)
        assert tokens[0] == first and lp[0] == 0.0, kw
    ref = _call(ppas, x, u=0.9)
    for kw in (dict(top_k=0), dict(top_k=-5), dict(top_k=5000), dict(top_k=2 ** 31 - 1), dict(top_p=1.0),
               dict(top_p=2.0), dict(top_p=math.nan), dict(min_p=0.0), dict(min_p=-1.0), dict(min_p=math.nan),
               dict(temperature=1.0)):
        assert _call(ppas, x, u=0.9, **kw) == ref, kw
    assert _call(ppas, x, u=-1.0) == _call(ppas, x, u=0.0)
    assert _call(ppas, x, u=math.nan) == _call(ppas, x, u=0.0)
    assert _call(ppas, x, u=1.0) == _call(ppas, x, u=50.0)
    assert _call(ppas, x, u=0.25, logprobs=False)[0] == _call(ppas, x, u=0.25)[0]


@pytest.mark.parametrize("bf16", [False, True])
def test_strides_and_alignment(ppas, bf16):
    """Rows at every offset from a 16-byte boundary give what contiguous ones do."""
    n, v = 9, 10007
    x = _logits(n, v, 6, bf16=bf16)
    rules = [RULES[r] for r in range(n)]
    u = np.random.default_rng(1).random(n).astype(np.float32)
    want = _call(ppas, x, *zip(*rules), u)
    for shift, gap in ((0, 1), (1, 0), (2, 3), (3, 5), (5, 8), (7, 1000)):
        base = torch.full((n * (v + gap) + shift + 16,), math.nan, dtype=x.dtype, device="cuda")
        y = base[shift:].as_strided((n, v), (v + gap, 1))
        y.copy_(x)
        got = _call(ppas, y, *zip(*rules), u)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1]), (shift, gap)


def test_rows_do_not_depend_on_the_batch(ppas):
    """The same row alone, in a small and in a large batch (other cluster sizes)."""
    x = _logits(160, 40000, 8)
    rules = [RULES[r % len(RULES)] for r in range(160)]
    u = np.random.default_rng(2).random(160).astype(np.float32)
    want = _call(ppas, x, *zip(*rules), u)
    for a, b in ((0, 1), (5, 6), (10, 14), (20, 60), (0, 100)):
        got = _call(ppas, x[a:b], *zip(*rules[a:b]), u[a:b])
        assert np.array_equal(got[0], want[0][a:b]) and np.array_equal(got[1], want[1][a:b])


def test_frequencies(ppas):
    """100,000 draws from 12 tokens: counts within 5 standard deviations."""
    n = 100000
    row = torch.tensor([0.3, -1.0, 2.0, 0.0, 1.5, -3.0, 0.7, 0.7, -math.inf, 1.0, 0.2, -0.5], device="cuda")
    x = row.repeat(n, 1)
    u = np.random.default_rng(3).random(n).astype(np.float32)
    tokens, _ = _call(ppas, x, 0.9, 8, 0.95, 0.0, u)
    order, w = so.candidates(row.cpu().numpy(), 0.9)
    total, kept = so.kept_weight(w, 8, 0.95, 0.0)
    p = np.zeros(12)
    p[order[:kept]] = w[:kept] / total
    got = np.bincount(tokens, minlength=12)
    assert np.all(np.abs(got - n * p) <= 5 * np.sqrt(n * p * (1 - p)) + 1e-9)


def test_streams_and_back_to_back(ppas):
    """On another stream, and many calls after one another that read what the
    kernel before them wrote."""
    x = _logits(4, 30000, 12)
    u = np.array([0.1, 0.4, 0.7, 0.95], np.float32)
    want = _call(ppas, x, 0.8, 50, 0.95, 0.0, u)
    side = torch.cuda.Stream()
    got = _call(ppas, x, 0.8, 50, 0.95, 0.0, u, stream=side)
    assert np.array_equal(got[0], want[0])
    y, d_u = torch.empty_like(x), torch.from_numpy(u).cuda()
    k = torch.full((4,), 50, dtype=torch.int32, device="cuda")
    outs = [torch.empty(4, dtype=torch.int32, device="cuda") for _ in range(20)]
    for i, o in enumerate(outs):
        torch.add(x, 0.0 if i % 2 else 1.0, out=y)
        if i % 2 == 0:
            y.neg_()
        ppas.ppas_sample_tokens(y, False, y.stride(0), 4, 30000, None, k, None, None, d_u, o)
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        z = x if i % 2 else -(x + 1.0)
        for r in range(4):
            assert int(o[r]) == _whole_numbers(z[r], 1.0, 50, 1.0, 0.0, u[r])
