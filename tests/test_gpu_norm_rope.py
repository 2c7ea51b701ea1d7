"""Head norms with rotary positions and KV append on the GPU, every element against
the float64 oracle.

Tolerance: one rounding to bf16 (2^-8 relative) of an fp32 result.  Before it, relative
to the sizes of the normalised pair: the angle 2^-25 turn (2e-7), sine, cosine and
products 4 roundings of 2^-24, the sum of squares at most 16 + 5 + 32 additions of positive
terms (53 2^-24, half of it after the root), the root's 2^-22 and two products: 3e-6."""
import numpy as np
import pytest
import torch

from oracle import norm
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
    t, h, d = shape
    base = wl.bf16_normal((t * (h * d + gap) + shift,), seed, "cuda")
    return base[shift:].as_strided((t, h, d), (h * d + gap, d, 1)), h * d + gap


class Step:
    def __init__(self, T, hq, hk, D, rotary, inter, seed, gap=0, shift=0, gain=1.0, weights=True, wshift=0, eps=1e-6,
                 factor=1.0):
        rng = np.random.default_rng(seed)
        self.T, self.hq, self.hk, self.D, self.rotary, self.inter = T, hq, hk, D, rotary, inter
        self.eps, self.factor = eps, factor
        self.q, self.qs = _rows((T, max(hq, 1), D), seed + 1, gap, shift)
        self.k, self.ks = _rows((T, hk, D), seed + 2, gap, shift)
        self.v, self.vs = _rows((T, hk, D), seed + 3, gap, shift)
        self.q.mul_(gain)
        self.k.mul_(gain)
        self.wq = self.wk = None
        if weights:
            w = torch.randn(2, D + wshift, generator=torch.Generator().manual_seed(seed)).cuda()
            self.wq, self.wk = w[0, wshift:], w[1].clone()[wshift:]
        self.blocks = -(-T // 16) + 3
        self.pos = rng.integers(-5, 131072, size=T).astype(np.int32)
        order = rng.permutation(self.blocks)
        self.slots = (order[np.arange(T) // 16] * 16 + np.arange(T) % 16).astype(np.int32)
        self.slots[rng.random(T) < 0.1] = -1
        self.freq = np.array([500000.0 ** (-2 * i / rotary) for i in range(rotary // 2)] or [0.0], np.float32)
        self.kc = torch.full((self.blocks, hk, 16, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.vc = torch.full_like(self.kc, 5.0)
        self.out = torch.full((T + 2, max(hq, 1), D), 3.0, dtype=torch.bfloat16, device="cuda")
        self.err = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.d_pos, self.d_slots, self.d_freq = (torch.from_numpy(x).cuda() for x in (self.pos, self.slots, self.freq))

    def args(self, **kw):
        a = dict(q=self.q, k=self.k, v=self.v, q_stride=self.qs, k_stride=self.ks, v_stride=self.vs,
                 d_q_weight=self.wq, d_k_weight=self.wk, eps=self.eps, d_positions=self.d_pos,
                 d_slot_mapping=self.d_slots, n_tokens=self.T, d_inv_freq=self.d_freq, rotary_dim=self.rotary,
                 interleaved=self.inter, factor=self.factor, q_out=self.out, k_cache=self.kc, v_cache=self.vc,
                 num_blocks=self.blocks, n_q_heads=self.hq, n_kv_heads=self.hk, head_dim=self.D, d_err_flag=self.err)
        a.update(kw)
        return a

    def _close(self, got, x, w, pos, what):
        y = norm.head_norm(x.double().cpu().numpy(), None if w is None else w.double().cpu().numpy(), float(
            np.float32(self.eps)))
        want = rope.rotate(y, pos, self.freq[:self.rotary // 2], self.rotary, self.inter, self.factor)
        r, size = self.rotary, np.abs(y)
        a, b = (y[..., 0:r:2], y[..., 1:r:2]) if self.inter else (y[..., :r // 2], y[..., r // 2:r])
        pair = (np.abs(a) + np.abs(b)) * abs(self.factor)
        if self.inter:
            size[..., 0:r:2] = size[..., 1:r:2] = pair
        else:
            size[..., :r // 2] = size[..., r // 2:r] = pair
        off = np.abs(got - want) - (2.0 ** -8 * np.abs(want) + 3e-6 * size + 1e-38)
        assert np.all(off <= 0), f"{what}: {off.max()}"

    def check(self, q0=None):
        torch.cuda.synchronize()
        assert int(self.err.item()) == 0
        if self.hq:
            self._close(self.out[:self.T].double().cpu().numpy(), self.q, self.wq, self.pos, "q")
        assert bool((self.out[self.T:] == 3.0).all())
        kc, vc = (x.transpose(1, 2).reshape(-1, self.hk, self.D).double().cpu().numpy() for x in (self.kc, self.vc))
        keep = self.slots >= 0
        self._close(kc[self.slots[keep]], self.k[torch.from_numpy(keep).cuda()], self.wk, self.pos[keep], "k")
        assert np.array_equal(vc[self.slots[keep]], self.v.double().cpu().numpy()[keep])
        free = np.ones(self.blocks * 16, bool)
        free[self.slots[keep]] = False
        assert np.all(kc[free] == 7.0) and np.all(vc[free] == 5.0)


@pytest.mark.parametrize("T", [1, 2, 17, 300, 2056])
@pytest.mark.parametrize("hq,hk", [(16, 2), (32, 8), (5, 1), (0, 3)])
@pytest.mark.parametrize("inter", [False, True])
def test_token_and_head_counts(ppas, T, hq, hk, inter):
    s = Step(T, hq, hk, 128, 128, inter, seed=T + hq, gap=(hq + hk) * 128)
    ppas.ppas_norm_rope_append(**s.args())
    s.check()


@pytest.mark.parametrize("D,rotary", [(128, 64), (128, 0), (64, 64), (256, 128), (512, 512), (80, 32), (80, 80), (24, 16),
                                      (8, 0), (136, 128), (8, 8), (128, 20), (24, 24), (80, 40), (504, 16)])
@pytest.mark.parametrize("inter", [False, True])
def test_head_and_rotary_sizes(ppas, D, rotary, inter):
    for T in (3, 70):
        s = Step(T, 6, 3, D, rotary, inter, seed=D + rotary + T, factor=1.25)
        ppas.ppas_norm_rope_append(**s.args())
        s.check()


@pytest.mark.parametrize("gap,shift,wshift", [(8, 0, 0), (3, 0, 0), (0, 1, 0), (0, 8, 4), (0, 0, 1), (1, 3, 3)])
@pytest.mark.parametrize("inter", [False, True])
def test_strides_and_alignment(ppas, gap, shift, wshift, inter):
    for T in (1, 40):
        s = Step(T, 16, 2, 128, 64, inter, seed=gap + shift, gap=gap, shift=shift, wshift=wshift)
        ppas.ppas_norm_rope_append(**s.args())
        s.check()


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("gain,eps", [(1e18, 1e-6), (1e30, 1e-6), (1e-3, 1e-6), (1e-20, 1e-6), (0.0, 1e-6), (1e-12, 1e-30),
                                      (1.0, 100.0)])
def test_sizes_of_activations(ppas, gain, eps, shift):
    """Squares past the fp32 range, heads of zeros, and an eps that counts."""
    s = Step(20, 4, 2, 128, 128, False, seed=3, gain=gain, eps=eps, shift=shift)
    ppas.ppas_norm_rope_append(**s.args())
    s.check()


@pytest.mark.parametrize("shift", [0, 1])
def test_one_large_head_among_ordinary_ones(ppas, shift):
    s = Step(33, 4, 2, 128, 128, False, seed=4, shift=shift)
    s.q[5, 2] *= 1e25
    s.k[7, 1] *= 3e37
    ppas.ppas_norm_rope_append(**s.args())
    s.check()


def test_no_weights_are_ones(ppas):
    for which in ("wq", "wk"):
        s = Step(20, 4, 2, 64, 32, True, seed=5)
        setattr(s, which, None)
        ppas.ppas_norm_rope_append(**s.args())
        s.check()


@pytest.mark.parametrize("rotary", [128, 20])
def test_in_place(ppas, rotary):
    s = Step(50, 16, 2, 128, rotary, False, seed=6)
    want = Step(50, 16, 2, 128, rotary, False, seed=6)
    ppas.ppas_norm_rope_append(**want.args())
    ppas.ppas_norm_rope_append(**s.args(q_out=s.q))
    torch.cuda.synchronize()
    assert torch.equal(s.q, want.out[:50]) and torch.equal(s.kc, want.kc)


def test_infinities_and_nan_stay_in_their_head(ppas):
    """A head with a NaN or an infinity spoils itself alone."""
    s = Step(9, 4, 2, 128, 128, False, seed=7)
    clean = Step(9, 4, 2, 128, 128, False, seed=7)
    s.q[3, 1, 5], s.q[4, 2, 7] = float("nan"), float("inf")
    for x in (s, clean):
        ppas.ppas_norm_rope_append(**x.args())
    torch.cuda.synchronize()
    same = torch.ones(9, 4, dtype=torch.bool)
    same[3, 1] = same[4, 2] = False
    assert torch.equal(s.out[:9][same.cuda()], clean.out[:9][same.cuda()]) and torch.equal(s.kc, clean.kc)
    assert bool(s.out[3, 1].isnan().all()) and bool(s.out[4, 2, [7, 71]].isnan().all())


def test_slot_past_the_cache_is_reported(ppas):
    for shift in (0, 1):
        s = Step(20, 4, 2, 128, 64, False, seed=8, shift=shift)
        s.slots[3] = s.blocks * 16
        s.d_slots = torch.from_numpy(s.slots).cuda()
        ppas.ppas_norm_rope_append(**s.args())
        torch.cuda.synchronize()
        assert int(s.err.item()) == ppas.PPAS_DEVERR_BAD_INDEX
        s.err.zero_()
        s.slots[3] = -1
        s.check()


def test_other_stream_and_graph(ppas):
    s = Step(64, 32, 8, 128, 128, False, seed=9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ppas.ppas_norm_rope_append(**s.args(stream=side))
    side.synchronize()
    s.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ppas.ppas_norm_rope_append(**s.args())
    s.q.mul_(-0.5)
    s.kc.fill_(7.0)
    graph.replay()
    s.check()


def test_past_32_bit_offsets(ppas):
    """Tokens' rows, and pages of the cache, further than 2^31 elements from the first."""
    T, hq, hk, D = 40, 4, 2, 128
    s = Step(T, hq, hk, D, 128, False, seed=10)
    stride = 1 << 26  # 40 * 2^26 > 2^31
    far = torch.empty((T, stride), dtype=torch.bfloat16, device="cuda")
    far[:, :hq * D] = s.q.reshape(T, hq * D)
    far[:, 1024:1024 + hk * D] = s.k.reshape(T, hk * D)
    far[:, 2048:2048 + hk * D] = s.v.reshape(T, hk * D)
    blocks = (1 << 31) // (hk * 16 * D) + 100
    kc = torch.zeros((blocks, hk, 16, D), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    slots = np.arange(T) + (blocks - 3) * 16
    want = Step(T, hq, hk, D, 128, False, seed=10)
    want.slots = np.arange(T, dtype=np.int32)
    want.d_slots = torch.from_numpy(want.slots).cuda()
    ppas.ppas_norm_rope_append(**want.args())
    ppas.ppas_norm_rope_append(**s.args(q=far, k=far[:, 1024:], v=far[:, 2048:], q_stride=stride, k_stride=stride,
                                        v_stride=stride, d_slot_mapping=torch.from_numpy(slots.astype(np.int32)).cuda(),
                                        k_cache=kc, v_cache=vc, num_blocks=blocks))
    torch.cuda.synchronize()
    assert int(s.err.item()) == 0 and torch.equal(s.out[:T], want.out[:T])
    assert torch.equal(kc[-3:, :, :].transpose(1, 2).reshape(-1, hk, D)[:T], want.kc.transpose(1, 2).reshape(-1, hk, D)[:T])
    assert torch.equal(vc[-3:, :, :].transpose(1, 2).reshape(-1, hk, D)[:T], want.vc.transpose(1, 2).reshape(-1, hk, D)[:T])


def test_cache_read_by_the_attention_step(ppas):
    """The next kernel of the stream reads what was appended, call after call without a wait."""
    hq, hk, D, T = 16, 2, 128, 64
    s = Step(T, hq, hk, D, 128, False, seed=11)
    s.slots = np.arange(T, dtype=np.int32)
    s.d_slots = torch.from_numpy(s.slots).cuda()
    s.kc.zero_()
    s.vc.zero_()
    table = torch.arange(4, dtype=torch.int32, device="cuda")[None]
    out = torch.empty((T, hq, D), dtype=torch.float32, device="cuda")

    def step(wait):
        ppas.ppas_norm_rope_append(**s.args())
        if wait:
            torch.cuda.synchronize()
        size = ppas.ppas_attention_workspace_size([T], [T], hq, hk)
        ws = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
        ppas.ppas_attention_step(s.out, s.kc, s.vc, s.blocks, table, 4, [T], [T], hq, hk, D, D ** -0.5, out, True, ws, size,
                                 s.err)
        torch.cuda.synchronize()
        return out.clone()
    want = step(True)
    for i in range(10):
        s.kc.fill_(float(i))
        s.vc.fill_(float(i))
        s.out.fill_(1.0)
        assert torch.equal(step(False), want)
