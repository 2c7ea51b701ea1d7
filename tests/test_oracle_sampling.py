"""The sampling oracle against closed forms and worked values, and the refusals
of the sampling call (CPU)."""
import numpy as np
import pytest

from oracle import sampling as so
from test_boundary_cpu import ppas  # noqa: F401

X = np.log([0.1, 0.4, 0.2, 0.05, 0.25])  # order 1, 4, 2, 0, 3


def test_inversion_over_the_order():
    for u, token in ((0.0, 1), (0.39, 1), (0.41, 4), (0.64, 4), (0.66, 2), (0.84, 2), (0.86, 0), (0.96, 3), (0.999, 3)):
        t, lp = so.sample(X, u=u)
        assert t == token and np.isclose(lp, X[token])


def test_cuts():
    # top-k 2: 0.4, 0.25 renormalised
    assert so.sample(X, top_k=2, u=0.62)[0] == 4 and so.sample(X, top_k=2, u=0.61)[0] == 1
    assert np.isclose(so.sample(X, top_k=2, u=0.62)[1], np.log(0.25 / 0.65))
    # top-p 0.64: two tokens reach 0.65; 0.66 takes a third
    assert so.kept_weight(so.candidates(X, 1.0)[1], 0, 0.64, 0.0)[1] == 2
    assert so.kept_weight(so.candidates(X, 1.0)[1], 0, 0.66, 0.0)[1] == 3
    # top-p of the three that top-k leaves: 0.4 / 0.85 = 0.47
    assert so.kept_weight(so.candidates(X, 1.0)[1], 3, 0.47, 0.0)[1] == 1
    assert so.kept_weight(so.candidates(X, 1.0)[1], 3, 0.48, 0.0)[1] == 2
    # min-p 0.3: 0.4, 0.25, 0.2 are at least 0.12
    assert so.kept_weight(so.candidates(X, 1.0)[1], 0, 1.0, 0.3)[1] == 3
    assert so.kept_weight(so.candidates(X, 1.0)[1], 0, 1.0, 2.0)[1] == 1
    assert so.kept_weight(so.candidates(X, 1.0)[1], 0, 0.0, 0.0)[1] == 1


def test_ties_temperature_and_empty_rows():
    assert so.sample([1.0, 3.0, 3.0, 3.0], top_k=2, u=0.99)[0] == 2
    assert so.sample([1.0, 3.0, 3.0], temperature=0.0) == (1, 0.0)
    order, w = so.candidates([0.0, -2.0], 2.0)
    assert np.allclose(w, [1, np.exp(-1)])
    assert so.sample([-np.inf, np.nan, -np.inf])[0] == -1
    assert so.sample([0.0, np.inf, 5.0, np.inf], u=0.7) == (3, np.log(0.5))
    assert so.sample([np.nan, 2.0], u=0.9)[0] == 1


def test_accepts_has_teeth():
    lp = X
    assert so.accepts(4, lp[4], X, 1.0, 0, 1.0, 0.0, 0.5, 1e-6)
    assert not so.accepts(1, lp[1], X, 1.0, 0, 1.0, 0.0, 0.5, 1e-6)
    assert so.accepts(1, lp[1], X, 1.0, 0, 1.0, 0.0, 0.4 + 1e-8, 1e-6)
    assert not so.accepts(4, lp[4] + 1e-3, X, 1.0, 0, 1.0, 0.0, 0.5, 1e-6)
    assert not so.accepts(2, lp[2], X, 1.0, 2, 1.0, 0.0, 0.99, 1e-6)


def test_refusals(ppas):  # noqa: F811
    ok = dict(logits=16, logits_are_bf16=False, row_stride=1000, n_rows=2, vocab=1000, d_temperature=16, d_top_k=16,
              d_top_p=16, d_min_p=16, d_uniform=16, d_tokens=16, d_logprobs=16, stream=0)
    for kw in (dict(n_rows=-1), dict(vocab=0), dict(row_stride=999), dict(logits=0), dict(d_uniform=0),
               dict(d_tokens=0), dict(logits=18), dict(logits=17, logits_are_bf16=True), dict(d_top_k=2),
               dict(d_logprobs=6)):
        with pytest.raises(ppas.PpasError) as e:
            ppas.ppas_sample_tokens(**{**ok, **kw})
        assert e.value.status == ppas.PPAS_ERR_INVALID_ARG, kw
    with pytest.raises(ppas.PpasError) as e:
        ppas.ppas_sample_tokens(**{**ok, "vocab": 262145, "row_stride": 262145})
    assert e.value.status == ppas.PPAS_ERR_UNSUPPORTED
    ppas.ppas_sample_tokens(**{**ok, "n_rows": 0, "logits": 0})  # no-op
