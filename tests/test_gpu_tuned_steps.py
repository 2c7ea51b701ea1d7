"""A batch whose iterations run out before its requests end."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_too_few_steps_are_an_error():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_15171_gb300 import tuned
    m = tuned.TunedDecoder(layers=1, vocab=500, inter=128, n_adapters=2, rank=8)
    requests = [tuned.Request(np.arange(30), 4, 0), tuned.Request(np.arange(9), 1, 1)]
    with pytest.raises(RuntimeError, match=r"\[0\] are unfinished"):
        tuned.Batch(m, requests).run(max_steps=3)
    assert len(requests[0].tokens) == 3 and len(requests[1].tokens) == 1
    done = tuned.Batch(m, [tuned.Request(np.arange(30), 4, 0), tuned.Request(np.arange(9), 1, 1)]).run(max_steps=4)
    assert [len(r.tokens) for r in done] == [4, 1]
