"""Requests of different adapters in one batch, end to end: the logits behind every
generated token, and the prompt's log probabilities, against a dense fp32 forward pass of each
request by itself, its adapter merged into the weights.

Tolerance: activations in bf16 (2^-9 of each, two layers of some fifteen roundings): a
relative error of the logits of a few times 2^-9 * sqrt(30) = 0.011, taken as 0.03 of their
norm; a prompt's log probability is off by what its logits are, 0.03 of their root mean square
of 2 units times a few (the largest of some hundred)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tuned():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_15171_gb300 import tuned as t
    return t


def _merged(w, adapters, which, scale):
    w = w.float()
    if which < 0:
        return w
    a, b, cols = adapters
    rank = b.shape[2]
    delta, at = [], 0
    for j, c in enumerate(cols.tolist()):
        delta.append(b[which, at:at + c].float() @ a[which, j * rank:(j + 1) * rank].float())
        at += c
    return w + scale * torch.cat(delta)


def _dense_logits(m, tokens, which):
    geo = m.geo
    hq, hk, d = geo.n_q_heads, geo.n_kv_heads, geo.head_dim
    t = tokens.numel()
    scale = float(m.scales[which]) if which >= 0 else 0.0
    x = m.embed[tokens].float()
    angle = torch.arange(t, device="cuda").double()[:, None] * m.inv_freq.double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]

    def norm(y):
        return y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6)

    def turn(y):
        a, b = y[..., :d // 2], y[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    causal = torch.ones(t, t, dtype=torch.bool, device="cuda").tril()
    for i in range(m.layers):
        w = _merged(m.w_qkv[i], m.qkv_adapters[i], which, scale)
        q, k, v = (norm(x) @ w.T).split([hq * d, hk * d, hk * d], dim=1)
        q = turn(norm(q.view(t, hq, d)) * m.q_norm[i])
        k = turn(norm(k.view(t, hk, d)) * m.k_norm[i])
        k, v = (y.repeat_interleave(hq // hk, dim=1) for y in (k, v.view(t, hk, d)))
        s = torch.einsum("qhd,khd->hqk", q, k) * geo.scale
        p = torch.softmax(s.masked_fill(~causal, float("-inf")), dim=-1)
        x = x + torch.einsum("hqk,khd->qhd", p, v).reshape(t, hq * d) @ _merged(m.w_o[i], m.o_adapters[i], which, scale).T
        gate, up = (norm(x) @ m.w_gate_up[i].float().T).chunk(2, dim=1)
        x = x + (torch.nn.functional.silu(gate) * up) @ _merged(m.w_down[i], m.down_adapters[i], which, scale).T
    return norm(x) @ m.w_out.float().T


@pytest.mark.parametrize("prompts,adapters,length,mbt", [
    ([40, 1, 130, 17], [0, -1, 2, 0], 6, 16384), ([700, 33, 400], [1, 1, -1], 4, 256), ([5] * 20, list(range(-1, 3)) * 5, 5, 64)])
def test_batches(tuned, prompts, adapters, length, mbt):
    m = tuned.TunedDecoder(layers=2, vocab=3001, inter=512, n_adapters=3, rank=8, seed=len(prompts))
    rng = np.random.default_rng(0)
    requests = [tuned.Request(rng.integers(0, m.vocab, size=n), length, a) for n, a in zip(prompts, adapters)]
    seen = {}
    tuned.Batch(m, requests, n_top=3, score_prompts=True, mbt_hi=mbt, mbt_lo=max(1, mbt // 2), seed=1).run(
        lambda r, place, x: seen.setdefault(r, []).append(x.clone()))
    for i, r in enumerate(requests):
        assert len(r.tokens) == length and len(seen[i]) == length
        every = torch.cat([torch.from_numpy(r.prompt), torch.tensor(r.tokens)]).cuda()
        want = _dense_logits(m, every, r.adapter)
        got = torch.stack(seen[i])
        behind = want[len(r.prompt) - 1:-1]
        assert float((got - behind).norm() / behind.norm()) < 0.03
        # what is reported is of the logits that were drawn from
        lp = torch.log_softmax(got.double(), dim=1)
        for j in range(length):
            assert abs(r.logprobs[j] - float(lp[j, r.tokens[j]])) < 2e-5
            assert abs(r.entropy[j] + float((lp[j].exp() * lp[j]).sum())) < 1e-4
            assert [t for t, _ in r.alternatives[j]] == torch.sort(got[j], descending=True, stable=True)[1][:3].tolist()
        assert len(r.prompt_logprobs) == len(r.prompt) - 1
        if len(r.prompt) > 1:
            lp = torch.log_softmax(want, dim=1)[torch.arange(len(r.prompt) - 1), every[1:len(r.prompt)]]
            off = (torch.tensor(r.prompt_logprobs).cuda() - lp).abs()
            assert float(off.max()) < 0.5 and float(off.mean()) < 0.1


def test_an_adapter_matters(tuned):
    m = tuned.TunedDecoder(layers=1, vocab=2000, inter=256, n_adapters=2, rank=8)
    prompt = np.arange(50)
    rules = tuned.answers.Rules(temperature=0.0)

    def tokens(ids):
        return [r.tokens for r in tuned.Batch(m, [tuned.Request(prompt, 6, a) for a in ids], rules).run()]
    together = tokens([0, -1, 1])
    assert together[0] != together[1] and together[1] != together[2] and together[0] != together[2]


def test_refusals(tuned):
    m = tuned.TunedDecoder(layers=1, vocab=100, inter=128, n_adapters=2, rank=8)
    for r in (tuned.Request(np.array([], np.int64), 3), tuned.Request(np.arange(3), 0), tuned.Request(np.arange(3), 2, 2)):
        with pytest.raises(ValueError):
            tuned.Batch(m, [r])
