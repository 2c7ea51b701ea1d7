"""Attention over shared prefixes on the GPU, every element against the float64
oracle row by row: group sizes from one row to several tiles, prefixes of a page
to several pieces, ragged ends, rows without own keys, groups without a prefix,
every geometry; slots outside every context hold NaN.  Closed forms for long
prefixes, the refused and damaged inputs, streams and back-to-back calls.

Tolerance: the weights of the weighted sum and the output are each rounded to
bf16 (2^-9 of themselves): the error's norm is at most 2^-9 (1 + 1) of the
result's, taken as 5e-3 with the fp32 rest; any element within the 2e-2 of the
ordinary step."""
import numpy as np
import pytest
import torch

from _cases import MAX_ABS, MEAN_ABS, host64
from oracle import attention as oa
from paper_2608_15171_gb300 import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ppas():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_15171_gb300 import ppas as p
    return p


class Batch:
    """Groups of rows with common prefix pages, own pages, NaN in every slot past a context."""

    def __init__(self, hq, hk, rows, prefixes, own, seed=0, gain=1.0, nan=True):
        rng = np.random.default_rng(seed)
        self.hq, self.hk, self.rows, self.prefixes = hq, hk, list(rows), list(prefixes)
        group = np.repeat(np.arange(len(rows)), rows)
        own = own if not np.isscalar(own) else [own] * len(group)
        self.ctx = [prefixes[g] + o for g, o in zip(group, own)]
        first = [p // 16 for p in prefixes]
        mine = [-(-c // 16) - first[g] for c, g in zip(self.ctx, group)]
        self.blocks = sum(first) + sum(mine) + 3
        order = rng.permutation(self.blocks).astype(np.int32)
        self.width = max(first[g] + m for g, m in zip(group, mine)) + 1
        self.table = np.full((len(group), self.width), -1, np.int32)
        at = 0
        shared = []
        for n in first:
            shared.append(order[at:at + n])
            at += n
        covered = np.zeros(self.blocks * 16, bool)
        for r, (g, m) in enumerate(zip(group, mine)):
            self.table[r, :first[g]] = shared[g]
            self.table[r, first[g]:first[g] + m] = order[at:at + m]
            at += m
            pos = np.arange(self.ctx[r])
            covered[self.table[r][pos // 16] * 16 + pos % 16] = True
        self.k = wl.bf16_normal((self.blocks, hk, 16, 128), seed * 7 + 1, "cuda")
        self.v = wl.bf16_normal((self.blocks, hk, 16, 128), seed * 7 + 2, "cuda")
        self.q = wl.bf16_normal((len(group), hq, 128), seed * 7 + 3, "cuda") * gain
        if nan:
            hole = torch.from_numpy(~covered).view(self.blocks, 1, 16, 1).cuda()
            self.k.masked_fill_(hole, float("nan"))
            self.v.masked_fill_(hole, float("nan"))
        self.n = len(group)
        self.d_table = torch.from_numpy(self.table).cuda()

    def call(self, ppas, stream=None, out=None, ws=None, sync=True, err=None, **kw):
        out = torch.full((self.n + 1, self.hq, 128), 3.0, dtype=torch.bfloat16, device="cuda") if out is None else out
        size = ppas.ppas_shared_attention_workspace_size(self.ctx, self.rows, self.prefixes, self.hq, self.hk)
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda") if ws is None else ws
        err = torch.zeros(1, dtype=torch.int32, device="cuda") if err is None else err
        if sync:
            torch.cuda.synchronize()
        a = dict(q=self.q, k_cache=self.k, v_cache=self.v, num_blocks=self.blocks, d_block_tables=self.d_table,
                 max_blocks_per_seq=self.width, ctx_lens=self.ctx, group_rows=self.rows, prefix_lens=self.prefixes,
                 n_q_heads=self.hq, n_kv_heads=self.hk, head_dim=128, scale=128 ** -0.5, out=out, workspace=ws,
                 workspace_bytes=size, d_err_flag=err, stream=stream)
        a.update(kw)
        ppas.ppas_shared_attention_step(**a)
        if sync:
            torch.cuda.synchronize()
            assert int(err.item()) == 0
            assert out.shape[0] == self.n or bool((out[self.n] == 3.0).all())
        return out[:self.n]

    def want(self):
        k, v = (torch.nan_to_num(x, nan=0.0) for x in (self.k, self.v))
        return oa.paged_attention(host64(self.q), host64(k), host64(v), self.table, [1] * self.n, self.ctx, 128 ** -0.5)

    def check(self, got, want=None):
        got, want = host64(got), self.want() if want is None else want
        assert np.all(np.isfinite(got))
        off = got - want
        assert np.abs(off).max() <= MAX_ABS and np.abs(off).mean() <= MEAN_ABS
        assert np.linalg.norm(off) <= 5e-3 * np.linalg.norm(want)


GEOMETRIES = [(16, 2), (32, 8), (8, 4), (8, 8), (4, 1)]


@pytest.mark.parametrize("hq,hk", GEOMETRIES)
@pytest.mark.parametrize("rows", [1, 2, 3, 15, 16, 17, 33, 40])
def test_rows_of_a_group(ppas, hq, hk, rows):
    b = Batch(hq, hk, [rows], [272], [1 + (r * 7) % 60 for r in range(rows)], seed=rows)
    b.check(b.call(ppas))


@pytest.mark.parametrize("rows,prefix", [(1, 4096), (1, 4112), (1, 9040), (2, 688), (2, 704), (2, 1040), (3, 1040),
                                         (8, 80), (8, 96), (8, 112)])
@pytest.mark.parametrize("hq,hk", GEOMETRIES)
def test_few_rows_of_a_prefix(ppas, rows, prefix, hq, hk):
    """Both sides of the lengths from which few rows read their prefix as one."""
    b = Batch(hq, hk, [rows, 1, rows], [prefix, 32, prefix + 16], [1 + 11 * r for r in range(2 * rows + 1)], seed=rows)
    b.check(b.call(ppas))


def test_long_own_keys(ppas):
    """One row's long context without a prefix, and beside rows with a few keys: many
    runs of one (row, kv-head), and runs of many."""
    b = Batch(16, 2, [1], [0], [30001], seed=20)
    b.check(b.call(ppas))
    b = Batch(16, 2, [3, 20], [64, 2048], [9000, 1, 0] + [r % 4 for r in range(20)], seed=21)
    b.check(b.call(ppas))


@pytest.mark.parametrize("prefix", [16, 32, 112, 128, 144, 256, 400, 512, 1024, 2000, 5008])
@pytest.mark.parametrize("hq,hk,rows", [(16, 2, 5), (32, 8, 40), (8, 8, 130)])
def test_prefix_lengths(ppas, prefix, hq, hk, rows):
    b = Batch(hq, hk, [rows], [prefix], [1 + r % 20 for r in range(rows)], seed=prefix)
    b.check(b.call(ppas))


@pytest.mark.parametrize("own", [0, 1, 15, 16, 17, 31, 32, 33, 64, 100, 511, 512, 513, 1500])
def test_own_lengths(ppas, own):
    for hq, hk in ((16, 2), (8, 8)):
        b = Batch(hq, hk, [6], [160], [own, max(own - 1, 0), own + 1, 0, own, 1], seed=own)
        b.check(b.call(ppas))


def test_no_own_keys_at_all(ppas):
    b = Batch(16, 2, [20, 4], [640, 16], 0, seed=1)
    b.check(b.call(ppas))


def test_no_prefix(ppas):
    b = Batch(16, 2, [3, 1], [0, 0], [1, 300, 17, 2000], seed=2)
    b.check(b.call(ppas))


@pytest.mark.parametrize("seed", range(6))
def test_several_groups(ppas, seed):
    rng = np.random.default_rng(seed)
    hq, hk = GEOMETRIES[seed % len(GEOMETRIES)]
    n = int(rng.integers(2, 9))
    rows = [int(x) for x in rng.choice([1, 2, 5, 17, 35], size=n)]
    pre = [int(x) * 16 for x in rng.integers(0, 90, size=n)]
    own = [int(x) for x in rng.integers(1, 200, size=sum(rows))]
    b = Batch(hq, hk, rows, pre, own, seed=seed)
    b.check(b.call(ppas))


def test_more_rows_and_groups_than_a_launch(ppas):
    """600 rows of one group, and 140 groups: several launches after one another."""
    b = Batch(8, 8, [600], [48], [1 + r % 5 for r in range(600)], seed=3)
    b.check(b.call(ppas))
    b = Batch(4, 1, [2] * 140, [32] * 140, [1 + r % 9 for r in range(280)], seed=4)
    b.check(b.call(ppas))


@pytest.mark.parametrize("gain", [4.0, 20.0])
def test_peaked_scores(ppas, gain):
    """Weights on a few keys, running maxima that grow along the prefix."""
    b = Batch(16, 2, [12], [1600], [1 + 3 * r for r in range(12)], seed=5, gain=gain)
    ramp = torch.linspace(0.2, 2.0, b.blocks, device="cuda").view(-1, 1, 1, 1)
    b.k.mul_(ramp[torch.argsort(torch.argsort(torch.arange(b.blocks, device="cuda")))])
    b.check(b.call(ppas))


def test_equals_the_ordinary_step(ppas):
    """The same rows through ppas_attention_step (as decode rows): within both roundings."""
    b = Batch(32, 8, [24], [3008], [5 + r for r in range(24)], seed=6)
    got = host64(b.call(ppas))
    out = torch.empty_like(b.q)
    size = ppas.ppas_attention_workspace_size([1] * b.n, b.ctx, 32, 8)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    ppas.ppas_attention_step(b.q, b.k, b.v, b.blocks, b.d_table, b.width, [1] * b.n, b.ctx, 32, 8, 128, 128 ** -0.5,
                             out, False, ws, size)
    torch.cuda.synchronize()
    assert np.abs(got - host64(out)).max() <= 2 * MAX_ABS
    assert np.linalg.norm(got - host64(out)) <= 1e-2 * np.linalg.norm(got)


def test_long_prefix_constant_values(ppas):
    """200,000 keys of one value and a NaN-free tail: the value comes back (to the
    rounding of the weights, 2^-8), over several pieces a CTA."""
    b = Batch(16, 2, [40], [200000], [1 + r % 30 for r in range(40)], seed=7)
    b.v.copy_(torch.where(torch.isnan(b.v), b.v, torch.full_like(b.v, 1.5)))
    got = host64(b.call(ppas))
    assert np.abs(got - 1.5).max() <= 1.5 * 2.0 ** -8


def test_prefix_longer_than_a_piece(ppas):
    """A prefix of over 512 KV tiles a piece on few SMs' worth of units: values
    that differ by half, against the exact mean of equal scores."""
    b = Batch(8, 8, [2], [16 * 40000], [1, 2], seed=8, nan=False)
    b.q.zero_()
    pages = torch.from_numpy(b.table[0, :40000]).cuda().long()
    b.v[pages[:20000]] = 1.0
    b.v[pages[20000:]] = 3.0
    got = host64(b.call(ppas))
    assert np.abs(got - 2.0).max() <= 2.0 * 2.0 ** -8


def test_single_key_and_same_rows(ppas):
    """One key in all: its value; equal rows of a group: equal results bit for bit."""
    b = Batch(16, 2, [1], [0], [1], seed=9)
    got = b.call(ppas)
    v = b.v[b.table[0, 0], :, 0].repeat_interleave(8, dim=0)
    assert torch.equal(got[0], v)
    b = Batch(16, 2, [40], [1024], 0, seed=10)
    b.q.copy_(b.q[:1].expand(40, -1, -1))
    got = b.call(ppas)
    assert torch.equal(got, got[:1].expand(40, -1, -1))


def test_bad_block_ids(ppas):
    for where in ("prefix", "own"):
        b = Batch(16, 2, [4], [256], [20] * 4, seed=11, nan=False)
        b.table[0 if where == "prefix" else 2, 3 if where == "prefix" else 17] = b.blocks if where == "own" else -5
        b.d_table = torch.from_numpy(b.table).cuda()
        err = torch.zeros(1, dtype=torch.int32, device="cuda")
        b.call(ppas, err=err, sync=False)
        torch.cuda.synchronize()
        assert int(err.item()) == ppas.PPAS_DEVERR_BAD_INDEX


def test_streams_and_back_to_back(ppas):
    """On another stream; calls that share a workspace after one another without
    a wait, each on the queries that the call before it wrote."""
    b = Batch(16, 2, [30], [1040], [1 + 5 * r for r in range(30)], seed=12)
    want = b.call(ppas)
    side = torch.cuda.Stream()
    assert torch.equal(b.call(ppas, stream=side), want)
    size = ppas.ppas_shared_attention_workspace_size(b.ctx, b.rows, b.prefixes, 16, 2)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    got = []
    for wait in (True, False):
        x, err = b.q.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        for _ in range(12):
            y = torch.empty_like(x)
            b.call(ppas, q=x, out=y, ws=ws, sync=wait, err=err)
            x = y
        torch.cuda.synchronize()
        got.append(x)
    assert torch.equal(got[0], got[1])


def test_graph_replay(ppas):
    """Captured once, replayed on new inputs."""
    b = Batch(16, 2, [20], [512], [1 + r for r in range(20)], seed=13)
    size = ppas.ppas_shared_attention_workspace_size(b.ctx, b.rows, b.prefixes, 16, 2)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    out, err = torch.empty_like(b.q), torch.zeros(1, dtype=torch.int32, device="cuda")
    b.call(ppas, out=out, ws=ws, err=err)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.call(ppas, out=out, ws=ws, sync=False, err=err)
    for s in range(3):
        b.q.copy_(wl.bf16_normal(tuple(b.q.shape), 50 + s, "cuda"))
        g.replay()
        torch.cuda.synchronize()
        b.check(out)
