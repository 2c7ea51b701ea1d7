"""Rotary positions with KV append on the GPU, every element against the float64
oracle: both layouts, all or part of the head, fused and odd strides, every
alignment, head sizes from 8 to 512, padded tokens, extreme positions, in place,
on another stream, and next to the attention step that reads the cache.

Tolerance: one rounding to bf16 (2^-8 relative) of an fp32 result whose angle is
off by at most 2^-25 turn and whose sine, cosine and products by a few units of
2^-24, all of the pair's size: 1e-6 of |a| + |b| times the factor."""
import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import rope
from paper_2608_15171_gb300 import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ppas():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_15171_gb300 import ppas as p
    return p


def _rows(shape, seed, gap, shift):
    """[T, heads, dim] with `gap` elements between rows, `shift` elements off a 256-byte boundary."""
    t, h, d = shape
    base = wl.bf16_normal((t * (h * d + gap) + shift,), seed, "cuda")
    return base[shift:].as_strided((t, h, d), (h * d + gap, d, 1)), h * d + gap


class Step:
    def __init__(self, T, hq, hk, D, rotary, inter, seed, gap=0, shift=0, positions=None, base=500000.0, factor=1.0):
        rng = np.random.default_rng(seed)
        self.T, self.hq, self.hk, self.D, self.rotary, self.inter, self.factor = T, hq, hk, D, rotary, inter, factor
        self.q, self.qs = _rows((T, max(hq, 1), D), seed + 1, gap, shift)
        self.k, self.ks = _rows((T, hk, D), seed + 2, gap, shift)
        self.v, self.vs = _rows((T, hk, D), seed + 3, gap, shift)
        self.blocks = -(-T // 16) + 3
        self.pos = rng.integers(0, 131072, size=T).astype(np.int32) if positions is None else positions
        order = rng.permutation(self.blocks)
        self.slots = (order[np.arange(T) // 16] * 16 + np.arange(T) % 16).astype(np.int32)
        self.slots[rng.random(T) < 0.1] = -1
        self.freq = np.array([base ** (-2 * i / rotary) for i in range(rotary // 2)] or [0.0], np.float32)
        self.kc = torch.full((self.blocks, hk, 16, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.vc = torch.full_like(self.kc, 5.0)
        self.out = torch.full((T + 2, max(hq, 1), D), 3.0, dtype=torch.bfloat16, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call(self, ppas, stream=None, **kw):
        a = dict(q=self.q, k=self.k, v=self.v, q_stride=self.qs, k_stride=self.ks, v_stride=self.vs,
                 d_positions=torch.from_numpy(self.pos).cuda(), d_slot_mapping=torch.from_numpy(self.slots).cuda(),
                 n_tokens=self.T, d_inv_freq=torch.from_numpy(self.freq).cuda(), rotary_dim=self.rotary,
                 interleaved=self.inter, factor=self.factor, q_out=self.out, k_cache=self.kc, v_cache=self.vc,
                 num_blocks=self.blocks, n_q_heads=self.hq, n_kv_heads=self.hk, head_dim=self.D,
                 d_err_flag=self.err, stream=stream)
        a.update(kw)
        ppas.ppas_rope_append(**a)
        torch.cuda.synchronize()

    def _close(self, got, x, what):
        x = x.double().cpu().numpy()
        want = rope.rotate(x, self.pos, self.freq[:self.rotary // 2], self.rotary, self.inter, self.factor)
        r, size = self.rotary, np.zeros_like(x)
        a, b = (x[..., 0:r:2], x[..., 1:r:2]) if self.inter else (x[..., :r // 2], x[..., r // 2:r])
        pair = (np.abs(a) + np.abs(b)) * abs(self.factor)
        if self.inter:
            size[..., 0:r:2] = size[..., 1:r:2] = pair
        else:
            size[..., :r // 2] = size[..., r // 2:r] = pair
        off = np.abs(got - want) - (2.0 ** -8 * np.abs(want) + 1e-6 * size)
        assert off.max() <= 0, f"{what}: {off.max()}"
        assert np.array_equal(got[..., r:], x[..., r:])

    def check(self, q_out=None):
        assert int(self.err.item()) == 0
        q_out = self.out if q_out is None else q_out
        if self.hq:
            self._close(q_out[:self.T].double().cpu().numpy(), self.q0 if hasattr(self, "q0") else self.q, "q")
        assert bool((self.out[self.T:] == 3.0).all())
        kc, vc = (x.transpose(1, 2).reshape(-1, self.hk, self.D).double().cpu().numpy() for x in (self.kc, self.vc))
        keep = self.slots >= 0
        got = np.zeros((self.T, self.hk, self.D))
        got[keep] = kc[self.slots[keep]]
        got[~keep] = rope.rotate(self.k.double().cpu().numpy()[~keep], self.pos[~keep], self.freq[:self.rotary // 2],
                                 self.rotary, self.inter, self.factor)
        self._close(got, self.k, "k") if not (~keep).any() else self._close_kept(got, keep)
        assert np.array_equal(vc[self.slots[keep]], self.v.double().cpu().numpy()[keep])
        free = np.ones(self.blocks * 16, bool)
        free[self.slots[keep]] = False
        assert np.all(kc[free] == 7.0) and np.all(vc[free] == 5.0)

    def _close_kept(self, got, keep):
        all_pos, self.pos = self.pos, self.pos[keep]
        self._close(got[keep], self.k[torch.from_numpy(keep).to(self.k.device)], "k")
        self.pos = all_pos


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 63, 300, 2056])
@pytest.mark.parametrize("hq,hk", [(16, 2), (32, 8), (8, 8), (5, 1)])
@pytest.mark.parametrize("inter", [False, True])
def test_token_and_head_counts(ppas, T, hq, hk, inter):
    s = Step(T, hq, hk, 128, 128, inter, seed=T + hq, gap=(hq + hk) * 128)
    s.call(ppas)
    s.check()


@pytest.mark.parametrize("D,rotary", [(128, 64), (128, 96), (128, 16), (128, 0), (64, 64), (64, 16), (256, 128),
                                      (512, 512), (512, 32), (80, 32), (80, 80), (96, 96), (24, 16), (8, 0), (136, 128),
                                      (8, 8), (128, 2), (128, 20), (64, 24), (24, 24), (80, 40)])
@pytest.mark.parametrize("inter", [False, True])
def test_head_and_rotary_sizes(ppas, D, rotary, inter):
    for T in (3, 70):
        s = Step(T, 6, 3, D, rotary, inter, seed=D + rotary + T, factor=1.25)
        s.call(ppas)
        s.check()


@pytest.mark.parametrize("gap,shift", [(8, 0), (3, 0), (0, 1), (1, 1), (0, 8), (4096, 16), (0, 4)])
@pytest.mark.parametrize("inter", [False, True])
def test_strides_and_alignment(ppas, gap, shift, inter):
    for T in (1, 40):
        s = Step(T, 16, 2, 128, 64, inter, seed=gap + shift, gap=gap, shift=shift)
        s.call(ppas)
        s.check()


def test_extreme_positions(ppas):
    """Angles of any 32-bit position are as good as those of small ones."""
    pos = np.array([0, 1, -1, 131071, 1 << 20, 10 ** 9, 2 ** 31 - 1, -2 ** 31, -12345, 7], np.int32)
    for inter in (False, True):
        for base in (10000.0, 500000.0, 1.0000001):
            s = Step(len(pos), 4, 2, 128, 128, inter, seed=1, positions=pos, base=base)
            s.call(ppas)
            s.check()


def test_odd_frequencies(ppas):
    """Frequencies above one, negative, zero, tiny and subnormal."""
    s = Step(20, 4, 2, 32, 32, False, seed=3)
    s.freq = np.array([100.5, -0.75, 0.0, 1e-12, 1e-38, 1e-42, 3.0e6, 1.0, 2 ** -20, -1e-5, 0.1, 0.2, 0.3, 0.4, 0.5,
                       6.2831855], np.float32)
    s.call(ppas)
    s.check()


@pytest.mark.parametrize("rotary", [128, 20])
@pytest.mark.parametrize("inter", [False, True])
def test_in_place(ppas, rotary, inter):
    s = Step(33, 16, 2, 128, rotary, inter, seed=5)
    s.q0 = s.q.clone()
    s.call(ppas, q_out=s.q)
    s.check(s.q)


def test_keys_and_values_alone(ppas):
    s = Step(33, 0, 2, 128, 128, False, seed=6)
    s.call(ppas, q=None, q_out=None, q_stride=0)
    s.check()


@pytest.mark.parametrize("rotary", [128, 20])
def test_slot_outside_the_cache(ppas, rotary):
    s = Step(18, 4, 2, 128, rotary, False, seed=7)
    s.slots[:] = np.arange(18)
    s.slots[4] = s.blocks * 16
    s.slots[9] = 2 ** 31 - 1
    s.call(ppas)
    assert int(s.err.item()) == ppas.PPAS_DEVERR_BAD_INDEX
    s.err.zero_()
    s.slots[4] = s.slots[9] = -1
    s.check()


def test_other_stream_and_no_flag(ppas):
    s = Step(64, 16, 2, 128, 128, False, seed=8)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s.call(ppas, d_err_flag=None)
    s.check()
    s.kc.fill_(7.0), s.vc.fill_(5.0)
    torch.cuda.synchronize()
    s.call(ppas, stream=side)
    s.check()


def test_wide_and_narrow_paths_agree(ppas):
    """The same rows 16 bytes and 2 bytes off alignment give the same bits."""
    a = Step(50, 16, 2, 128, 64, True, seed=9, gap=8, shift=0)
    b = Step(50, 16, 2, 128, 64, True, seed=9, gap=9, shift=1)
    for n in ("q", "k", "v"):
        getattr(b, n).copy_(getattr(a, n))
    a.call(ppas)
    b.call(ppas)
    assert torch.equal(a.out, b.out) and torch.equal(a.kc, b.kc) and torch.equal(a.vc, b.vc)


def test_append_then_attention(ppas):
    """Back to back on one stream, many times: the step reads what the append
    before it wrote; against the oracle on rotated inputs."""
    T, hq, hk, D = 40, 16, 2, 128
    rng = np.random.default_rng(10)
    blocks = 8
    freq = torch.tensor([10000.0 ** (-i / 64) for i in range(64)], dtype=torch.float32).cuda()
    table = rng.permutation(blocks)[:3].astype(np.int32)[None]
    slots = (table[0][np.arange(T) // 16] * 16 + np.arange(T) % 16).astype(np.int32)
    kc = torch.zeros((blocks, hk, 16, D), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    d_slots, d_table = torch.from_numpy(slots).cuda(), torch.from_numpy(table).cuda()
    d_pos = torch.arange(T, dtype=torch.int32, device="cuda")
    ws_bytes = ppas.ppas_attention_workspace_size([T], [T], hq, hk)
    ws = torch.empty(max(ws_bytes, 256), dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    ins = [wl.bf16_normal((T, (hq + 2 * hk) * D), 20 + i, "cuda") for i in range(6)]
    qr = torch.empty((T, hq, D), dtype=torch.bfloat16, device="cuda")
    outs = [torch.empty((T, hq, D), dtype=torch.float32, device="cuda") for _ in ins]
    torch.cuda.synchronize()
    for x, out in zip(ins, outs):
        q, k, v = x.split([hq * D, hk * D, hk * D], dim=1)
        n = x.stride(0)
        ppas.ppas_rope_append(q, k, v, n, n, n, d_pos, d_slots, T, freq, D, False, 1.0, qr, kc, vc, blocks, hq, hk, D,
                              err)
        ppas.ppas_attention_step(qr, kc, vc, blocks, d_table, 3, [T], [T], hq, hk, D, D ** -0.5, out, True, ws,
                                 ws_bytes, err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    f = freq.cpu().numpy()
    for x, out in zip(ins, outs):
        q, k, v = (y.reshape(T, -1, D).double().cpu().numpy() for y in x.split([hq * D, hk * D, hk * D], dim=1))
        kh, vh = np.zeros((blocks, hk, 16, D)), np.zeros((blocks, hk, 16, D))
        oa.kv_append(rope.rotate(k, np.arange(T), f, D, False), v, slots, kh, vh)
        want = oa.paged_attention(rope.rotate(q, np.arange(T), f, D, False), kh, vh, table, [T], [T], D ** -0.5)
        off = np.abs(out.double().cpu().numpy() - want)
        assert off.max() <= 4e-2 and off.mean() <= 3e-3  # the step's own 2e-2 and 2e-3, and q, k rounded to bf16
