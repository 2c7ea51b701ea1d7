"""Rotary positions on the host: the frequencies of each scaling against their
definitions, the oracle against closed forms, and the refusals of the append."""
import math

import numpy as np
import pytest

from oracle import rope
from test_boundary_cpu import ppas  # noqa: F401


@pytest.mark.parametrize("name,args", [
    ("plain", ()), ("linear", (4.0,)), ("base", (8.0,)),
    ("bands", (8.0, 8192, 1.0, 4.0)), ("bands", (1.0, 4096, 1.0, 4.0)), ("bands", (32.0, 131072, 0.5, 16.0)),
    ("ramp", (4.0, 4096, 1.0, 32.0)), ("ramp", (40.0, 32768, 1.0, 32.0)), ("ramp", (2.0, 64, 1.0, 32.0)),
])
@pytest.mark.parametrize("rotary,base", [(128, 500000.0), (64, 10000.0), (20, 1000000.0), (4, 10000.0)])
def test_frequencies(ppas, name, args, rotary, base):  # noqa: F811
    kind = {"plain": ppas.PPAS_ROPE_PLAIN, "linear": ppas.PPAS_ROPE_LINEAR, "base": ppas.PPAS_ROPE_BASE,
            "bands": ppas.PPAS_ROPE_BANDS, "ramp": ppas.PPAS_ROPE_RAMP}[name]
    got, factor = ppas.ppas_rope_frequencies(kind, rotary, base, *args)
    want, want_factor = rope.frequencies(name, rotary, base, *args)
    # one rounding to fp32 of doubles that agree to a few units in the last place
    assert got.dtype == np.float32 and got.shape == (rotary // 2,)
    assert np.max(np.abs(got.astype(np.float64) / np.array(want) - 1)) <= 2 ** -24 + 1e-12
    assert abs(factor - want_factor) <= 2 ** -23 * want_factor


def test_frequencies_worked_values(ppas):  # noqa: F811
    f, factor = ppas.ppas_rope_frequencies(ppas.PPAS_ROPE_PLAIN, 8, 10000.0)
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001], rtol=1e-7) and factor == 1.0
    f, _ = ppas.ppas_rope_frequencies(ppas.PPAS_ROPE_LINEAR, 8, 10000.0, 4.0)
    assert np.allclose(f, [0.25, 0.025, 0.0025, 0.00025], rtol=1e-7)
    # the slowest pair of a scaled base has its wavelength stretched by the scale
    f, _ = ppas.ppas_rope_frequencies(ppas.PPAS_ROPE_BASE, 8, 10000.0, 4.0)
    assert f[0] == 1.0 and np.isclose(f[3], 0.001 / 4, rtol=1e-6)
    # 8192 positions: wavelengths under 2048 kept, over 8192 stretched
    f, _ = ppas.ppas_rope_frequencies(ppas.PPAS_ROPE_BANDS, 128, 500000.0, 8.0, 8192, 1.0, 4.0)
    plain, _ = ppas.ppas_rope_frequencies(ppas.PPAS_ROPE_PLAIN, 128, 500000.0)
    wave = 2 * math.pi / plain.astype(np.float64)
    assert np.array_equal(f[wave < 2047], plain[wave < 2047])
    assert np.allclose(f[wave > 8193], plain[wave > 8193] / 8, rtol=1e-6)
    assert np.all(np.diff(f) < 0)


def test_frequency_refusals(ppas):  # noqa: F811
    for args in ((0, 7, 1e4), (0, 0, 1e4), (0, 128, 1.0), (0, 128, float("nan")), (5, 128, 1e4), (-1, 128, 1e4),
                 (1, 128, 1e4, 0.5), (1, 128, 1e4, float("inf")), (2, 2, 1e4, 2.0), (3, 128, 1e4, 8.0, 0, 1.0, 4.0),
                 (3, 128, 1e4, 8.0, 8192, 4.0, 4.0), (4, 128, 1e4, 8.0, 8192, 0.0, 4.0)):
        with pytest.raises(ppas.PpasError) as e:
            ppas.ppas_rope_frequencies(*args)
        assert e.value.status == ppas.PPAS_ERR_INVALID_ARG, args


def test_oracle_closed_forms():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 3, 12))
    f = [1.0, 0.25, 0.0]
    # position 0 and frequency 0 leave a pair alone; norms of pairs are kept
    assert np.array_equal(rope.rotate(x, [0] * 5, f, 6, False), x)
    y = rope.rotate(x, [3, 1, 4, 1, 5], f, 6, False)
    assert np.allclose(y[..., 2], x[..., 2]) and np.allclose(y[..., 5], x[..., 5])
    assert np.allclose(y[..., 0] ** 2 + y[..., 3] ** 2, x[..., 0] ** 2 + x[..., 3] ** 2)
    assert np.array_equal(y[..., 6:], x[..., 6:])
    # a quarter turn: (a, b) -> (-b, a)
    z = rope.rotate(x[:1], [1], [math.pi / 2], 2, True)
    assert np.allclose(z[..., 0], -x[:1, :, 1]) and np.allclose(z[..., 1], x[:1, :, 0])
    # the layouts are one another's permutation
    perm = [0, 2, 4, 1, 3, 5, 6, 7, 8, 9, 10, 11]
    half = rope.rotate(x[..., perm], [9] * 5, f, 6, False)
    assert np.allclose(half, rope.rotate(x, [9] * 5, f, 6, True)[..., perm])
    # scores depend on the distance of positions alone
    a, b = rng.standard_normal((1, 1, 6)), rng.standard_normal((1, 1, 6))

    def score(s, t):
        return float(np.sum(rope.rotate(a, [s], f, 6, False) * rope.rotate(b, [t], f, 6, False)))
    assert abs(score(7, 3) - score(1004, 1000)) < 1e-9


def test_append_refusals(ppas):  # noqa: F811
    ok = dict(q=16, k=16, v=16, q_stride=2560, k_stride=2560, v_stride=2560, d_positions=16, d_slot_mapping=16,
              n_tokens=3, d_inv_freq=16, rotary_dim=128, interleaved=False, factor=1.0, q_out=4096, k_cache=16,
              v_cache=16, num_blocks=4, n_q_heads=16, n_kv_heads=2, head_dim=128, stream=0)
    bad = [dict(n_tokens=-1), dict(head_dim=12), dict(head_dim=4), dict(num_blocks=0), dict(n_kv_heads=0),
           dict(n_q_heads=-1), dict(rotary_dim=-2), dict(rotary_dim=7), dict(rotary_dim=130),
           dict(factor=float("nan")), dict(q_stride=2047), dict(k_stride=255), dict(v_stride=-256), dict(q=0),
           dict(k=0), dict(v=0), dict(d_positions=0), dict(d_slot_mapping=0), dict(d_inv_freq=0), dict(q_out=0),
           dict(k_cache=0), dict(v_cache=0), dict(q=17), dict(k_cache=24), dict(d_positions=18),
           dict(q=4096)]  # in place, with a stride that is not the output's
    for kw in bad:
        with pytest.raises(ppas.PpasError) as e:
            ppas.ppas_rope_append(**{**ok, **kw})
        assert e.value.status == ppas.PPAS_ERR_INVALID_ARG, kw
    for kw in (dict(head_dim=520, rotary_dim=0, q_stride=1 << 20, k_stride=1 << 20, v_stride=1 << 20),
               dict(num_blocks=1 << 27), dict(n_q_heads=65537, q_stride=1 << 40)):
        with pytest.raises(ppas.PpasError) as e:
            ppas.ppas_rope_append(**{**ok, **kw})
        assert e.value.status == ppas.PPAS_ERR_UNSUPPORTED, kw
    ppas.ppas_rope_append(**{**ok, "n_tokens": 0, "q": 0})  # no-op
