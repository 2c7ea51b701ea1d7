"""The answers example end to end: the tokens it draws and the logits it draws
them from, against a dense fp32 forward pass over prompt and answer together.

Tolerance: the loop's activations are bf16 (2^-9 of each, two layers of a dozen
roundings) and its attention weights too: a relative error of the logits of a few
times 2^-9 * sqrt(24) = 0.01, taken as 0.03 of their norm."""
import numpy as np
import pytest
import torch

from oracle import sampling as so

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def answers():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_15171_gb300 import answers as a
    return a


def _dense_logits(m, tokens):
    """Logits after every token of one sequence, fp32, no cache and no kernels of the library."""
    geo = m.geo
    hq, hk, d = geo.n_q_heads, geo.n_kv_heads, geo.head_dim
    t = tokens.numel()
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
        q, k, v = (norm(x) @ m.w_qkv[i].float().T).split([hq * d, hk * d, hk * d], dim=1)
        q, k, v = turn(q.view(t, hq, d)), turn(k.view(t, hk, d)), v.view(t, hk, d)
        k, v = (y.repeat_interleave(hq // hk, dim=1) for y in (k, v))
        s = torch.einsum("qhd,khd->hqk", q, k) * geo.scale
        w = torch.softmax(s.masked_fill(~causal, float("-inf")), dim=-1)
        x = x + torch.einsum("hqk,khd->qhd", w, v).reshape(t, hq * d) @ m.w_o[i].float().T
        gate, up = (norm(x) @ m.w_gate_up[i].float().T).chunk(2, dim=1)
        x = x + (torch.nn.functional.silu(gate) * up) @ m.w_down[i].float().T
    return norm(x) @ m.w_out.float().T


@pytest.mark.parametrize("p_len,n,length", [(160, 5, 20), (167, 12, 12), (5, 3, 30), (1000, 2, 6)])
def test_answers(answers, p_len, n, length):
    m = answers.Decoder(layers=2, vocab=3001, inter=512, seed=p_len)
    prompt = np.random.default_rng(1).integers(0, m.vocab, size=p_len)
    seen = []
    rules = answers.Rules(0.9, 200, 0.95, 0.01)
    tokens, logprobs = answers.generate(m, prompt, n, length, rules, seed=3,
                                        on_step=lambda i, x, u, t: seen.append((x.clone(), u.clone(), t.clone())))
    assert tokens.shape == (n, length) and int(tokens.min()) >= 0 and int(tokens.max()) < m.vocab
    assert len({tuple(r) for r in tokens.tolist()}) > 1  # the answers differ
    for r in range(n):
        want = _dense_logits(m, torch.cat([torch.from_numpy(prompt).cuda(), tokens[r].long()]))[p_len - 1:-1]
        got = torch.stack([x[r] for x, _, _ in seen])
        assert float((got - want).norm() / want.norm()) < 0.03
    f32 = np.float32
    for i, (x, u, t) in enumerate(seen):
        assert torch.equal(t, tokens[:, i])
        for r in range(n):
            assert so.accepts(int(t[r]), float(logprobs[r, i]), x[r].cpu().numpy(), float(f32(0.9)), 200,
                              float(f32(0.95)), float(f32(0.01)), float(u[r]), 1e-5)


def test_same_seed_same_answers(answers):
    m = answers.Decoder(layers=1, vocab=2000, inter=256)
    prompt = list(range(50))
    a = answers.generate(m, prompt, 7, 9, seed=5)
    b = answers.generate(m, prompt, 7, 9, seed=5)
    c = answers.generate(m, prompt, 7, 9, seed=6)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and not torch.equal(a[0], c[0])


def test_greedy_answers_are_one(answers):
    m = answers.Decoder(layers=1, vocab=2000, inter=256)
    t, lp = answers.generate(m, list(range(33)), 4, 8, answers.Rules(temperature=0.0))
    assert torch.equal(t, t[:1].expand(4, -1)) and bool((lp == 0).all())


def test_refusals(answers):
    m = answers.Decoder(layers=1, vocab=100, inter=128)
    with pytest.raises(ValueError):
        answers.Answers(m, [], 2, 3)
    run = answers.Answers(m, [1, 2, 3], 2, 3)
    with pytest.raises(ValueError):
        run.step(torch.zeros(2, dtype=torch.int32, device="cuda"), 3)
