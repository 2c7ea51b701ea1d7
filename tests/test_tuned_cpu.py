"""What a batch of differently fine-tuned requests refuses, and that it does not return
unfinished ones (CPU only: a model without layers, no iteration is run)."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2608_15171_gb300 import workloads as wl
from test_boundary_cpu import ppas  # noqa: F401


@pytest.fixture(scope="module")
def tuned(ppas):  # noqa: F811
    from paper_2608_15171_gb300 import tuned as t
    return t


def _model():
    return SimpleNamespace(geo=wl.QWEN25_3B, layers=0, vocab=100, n_adapters=2, embed=torch.zeros(100, 8))


def test_unfinished_requests_are_an_error(tuned):
    batch = tuned.Batch(_model(), [tuned.Request(np.arange(5), 3)])
    with pytest.raises(RuntimeError, match="unfinished"):
        batch.run(max_steps=0)


def test_an_empty_plan_with_requests_left_is_an_error(tuned, monkeypatch):
    monkeypatch.setattr(tuned.ppas.Scheduler, "plan", lambda self, *a: SimpleNamespace(n_rows=0))
    batch = tuned.Batch(_model(), [tuned.Request(np.arange(5), 3), tuned.Request(np.arange(2), 1)])
    with pytest.raises(RuntimeError, match="unfinished"):
        batch.run()


def test_requests_that_have_run_or_come_twice_are_refused(tuned):
    """Tokens are appended to a request as they are drawn: each may be in one batch, once."""
    fresh, ran, scored = (tuned.Request(np.arange(5), 3) for _ in range(3))
    ran.tokens.append(1)
    scored.prompt_logprobs.append(-1.0)
    for requests in ([fresh, ran], [scored], [fresh, fresh]):
        with pytest.raises(ValueError):
            tuned.Batch(_model(), requests)
    batch = tuned.Batch(_model(), [fresh])
    fresh.tokens.append(1)
    with pytest.raises(ValueError):
        batch.run(max_steps=0)


def test_tokens_outside_the_vocabulary_are_refused(tuned):
    """Before they index the embedding on the device."""
    for prompt in ([5, 100], [-1, 3], [2 ** 31, 0], [0.5, 1.0], [[1, 2], [3, 4]]):
        with pytest.raises(ValueError):
            tuned.Batch(_model(), [tuned.Request(np.array(prompt), 2)])
    with np.errstate(invalid="ignore"), pytest.raises(ValueError):
        tuned.Batch(_model(), [tuned.Request(np.array([0.0, np.nan]), 2)])
    # whole numbers of any type are tokens
    tuned.Batch(_model(), [tuned.Request(np.array([0, 99], dtype), 2) for dtype in (np.int32, np.int64, np.uint8, float)])
    tuned.Batch(_model(), [tuned.Request([0, 99], 2), tuned.Request(torch.tensor([5]), 2)])
