"""Refusals of the head norms with append, the adapters and the log probabilities, and
the oracles against closed forms (CPU only: no call reaches a kernel)."""
import math

import numpy as np
import pytest

from oracle import adapter as oad
from oracle import logprobs as ol
from oracle import norm
from test_boundary_cpu import ppas  # noqa: F401


def _refused(call, ok, bad, status, error):
    for kw in bad:
        with pytest.raises(error) as e:
            call(**{**ok, **kw})
        assert e.value.status == status, kw


def test_norm_rope_refusals(ppas):  # noqa: F811
    ok = dict(q=16, k=16, v=16, q_stride=2560, k_stride=2560, v_stride=2560, d_q_weight=16, d_k_weight=0, eps=1e-6,
              d_positions=16, d_slot_mapping=16, n_tokens=3, d_inv_freq=16, rotary_dim=128, interleaved=False,
              factor=1.0, q_out=4096, k_cache=16, v_cache=16, num_blocks=4, n_q_heads=16, n_kv_heads=2, head_dim=128,
              stream=0)
    bad = [dict(n_tokens=-1), dict(head_dim=12), dict(num_blocks=0), dict(n_kv_heads=0), dict(rotary_dim=7),
           dict(factor=float("inf")), dict(q_stride=2047), dict(q=0), dict(v=0), dict(d_inv_freq=0), dict(k_cache=24),
           dict(q=4096), dict(eps=0.0), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")),
           dict(d_q_weight=18), dict(d_k_weight=1)]
    _refused(ppas.ppas_norm_rope_append, ok, bad, ppas.PPAS_ERR_INVALID_ARG, ppas.PpasError)
    bad = [dict(head_dim=520, rotary_dim=0, q_stride=1 << 20, k_stride=1 << 20, v_stride=1 << 20),
           dict(num_blocks=1 << 27)]
    _refused(ppas.ppas_norm_rope_append, ok, bad, ppas.PPAS_ERR_UNSUPPORTED, ppas.PpasError)
    ppas.ppas_norm_rope_append(**{**ok, "n_tokens": 0, "q": 0})  # no-op


def test_adapter_refusals(ppas):  # noqa: F811
    ok = dict(x=16, x_stride=256, y=1 << 20, y_stride=192, out=1 << 21, out_stride=192, q_lens=[1, 3], adapters=[0, -1],
              a=16, b=16, d_scales=16, n_adapters=2, hidden=256, slice_cols=[128, 64], rank=16, stream=0)
    bad = [dict(x=0), dict(y=0), dict(out=0), dict(a=0), dict(b=0), dict(x=18), dict(out=24), dict(d_scales=18),
           dict(x_stride=248), dict(y_stride=184), dict(out_stride=184), dict(x_stride=260), dict(q_lens=[0, 3]),
           dict(q_lens=[1, -3]), dict(adapters=[2, 0]), dict(adapters=[-2, 0]), dict(n_adapters=0), dict(hidden=0),
           dict(rank=0), dict(slice_cols=[]), dict(slice_cols=[128, 0]), dict(out=1 << 20, out_stride=200),
           dict(out=16), dict(adapters=[0]), dict(d_err_flag=3)]
    _refused(ppas.ppas_adapter_add, ok, bad, ppas.PPAS_ERR_INVALID_ARG, ppas.PpasError)
    bad = [dict(hidden=252, x_stride=256), dict(rank=12), dict(rank=136), dict(slice_cols=[128, 60]),
           dict(slice_cols=[8] * 5), dict(x_stride=1 << 37), dict(q_lens=[1 << 24, 1]), dict(n_adapters=1 << 27),
           dict(slice_cols=[1 << 24, 8], y_stride=1 << 25, out_stride=1 << 25)]
    _refused(ppas.ppas_adapter_add, ok, bad, ppas.PPAS_ERR_UNSUPPORTED, ppas.PpasError)
    ppas.ppas_adapter_add(**{**ok, "q_lens": [], "adapters": [], "x": 0})  # no-op
    # nobody has an adapter and the rows are where they belong: nothing to do
    ppas.ppas_adapter_add(**{**ok, "adapters": [-1, -1], "out": 1 << 20})


def test_logprob_refusals(ppas):  # noqa: F811
    ok = dict(logits=16, logits_are_bf16=False, row_stride=1000, n_rows=2, vocab=1000, d_tokens=16, d_logprobs=16,
              d_entropy=0, n_top=3, d_top_tokens=16, d_top_logprobs=16, stream=0)
    bad = [dict(n_rows=-1), dict(vocab=0), dict(n_top=-1), dict(row_stride=999), dict(logits=0), dict(d_tokens=0),
           dict(d_logprobs=0), dict(d_top_tokens=0), dict(d_top_logprobs=0), dict(logits=18), dict(d_tokens=17),
           dict(d_entropy=2), dict(n_top=0, d_tokens=0, d_logprobs=0), dict(logits=17, logits_are_bf16=True)]
    _refused(ppas.ppas_token_logprobs, ok, bad, ppas.PPAS_ERR_INVALID_ARG, ppas.PpasError)
    bad = [dict(vocab=262145, row_stride=300000), dict(n_top=33), dict(n_rows=1 << 28)]
    _refused(ppas.ppas_token_logprobs, ok, bad, ppas.PPAS_ERR_UNSUPPORTED, ppas.PpasError)
    ppas.ppas_token_logprobs(**{**ok, "n_rows": 0, "logits": 0})  # no-op


def test_norm_closed_forms():
    x = np.array([[[3.0, 4.0, 0.0, 0.0]]])
    assert np.allclose(norm.head_norm(x, None, 0.0), x / 2.5)  # mean square 25 / 4
    assert np.allclose(norm.head_norm(x * 7, [1.0, 2.0, 3.0, 4.0], 0.0), [[[1.2, 3.2, 0.0, 0.0]]])
    assert np.allclose(norm.head_norm(x, None, 18.75), x / 5)


def test_adapter_closed_forms():
    rng = np.random.default_rng(0)
    x, y = rng.normal(size=(3, 8)), rng.normal(size=(3, 16))
    a, b = rng.normal(size=(2, 16, 8)), rng.normal(size=(2, 16, 8))
    got = oad.adapter_add(x, y, [1, 2], [-1, 1], a, b, [5.0, 2.0], [8, 8], 8)
    assert np.array_equal(got[0], y[0])
    # the whole weight of an adapter, written out
    for c in range(16):
        j = c // 8
        w = sum(b[1, c, r] * a[1, j * 8 + r] for r in range(8))
        assert np.allclose(got[1:, c], y[1:, c] + 2.0 * x[1:] @ w)


def test_logprob_closed_forms():
    big = float(np.finfo(np.float32).max)
    lp, ent, tok, top = ol.row([0.0] * 8, 3, 10, big)
    assert np.isclose(lp, -math.log(8)) and np.isclose(ent, math.log(8))
    assert tok.tolist() == [0, 1, 2, 3, 4, 5, 6, 7, -1, -1] and top[8] == -np.inf
    lp, ent, tok, top = ol.row([-np.inf, math.log(0.25), np.nan, math.log(0.75)], 1, 3, big)
    assert np.isclose(lp, math.log(0.25)) and tok.tolist() == [3, 1, -1]
    assert np.isclose(ent, -(0.25 * math.log(0.25) + 0.75 * math.log(0.75)))
    assert ol.row([-np.inf] * 4, 2, 1, big)[:2] == (-np.inf, 0.0) and ol.row([1.0, np.inf], -1, 0, big)[0] == 0.0
