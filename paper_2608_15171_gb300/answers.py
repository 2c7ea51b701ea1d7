"""Several answers to one prompt, sampled side by side: the decode loop that the
rotary append, the attention over shared prefixes and the sampler are made for,
on a small decoder with random weights (there are no checkpoints here).

The prompt is computed once (``ppas_rope_append`` into the paged cache and
``ppas_attention_step`` chunk by chunk).  Its whole pages are then shared by all
answers; the last page, when it is not full, is copied for each of them.  Every
iteration takes one token of every answer through the layers

    q, k, v = norm(x) W_qkv        ppas_rope_append: rotated, keys and values appended
    x += attention W_o             ppas_shared_attention_step: the prompt read once for all answers
    x += gated MLP(norm(x))        ppas_gateup_swiglu

and draws the next ones from the logits (``ppas_sample_tokens``).  Norms and the
plain matrix products are torch's.

    python -m paper_2608_15171_gb300.answers --prompt 25000 --answers 32 --tokens 16
"""
from __future__ import annotations

import argparse
import math
from dataclasses import dataclass

import numpy as np
import torch

from . import ppas
from . import workloads as wl

PAGE = wl.PAGE_TOKENS


@dataclass
class Rules:
    """How the next tokens are drawn (one set of rules for all answers)."""
    temperature: float = 0.8
    top_k: int = 0
    top_p: float = 0.95
    min_p: float = 0.0


class Decoder:
    """A decoder of ``layers`` layers with seeded random weights in bf16."""

    def __init__(self, geo: wl.Geometry = wl.QWEN25_3B, layers: int = 2, vocab: int = 32000, inter: int = 4096,
                 seed: int = 0, device="cuda"):
        self.geo, self.layers, self.vocab, self.inter = geo, layers, vocab, inter
        d, hq, hk = geo.head_dim, geo.n_q_heads, geo.n_kv_heads
        self.hidden = hq * d
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(rows, cols):
            return (torch.randn(rows, cols, generator=g, device=device) / math.sqrt(cols)).to(torch.bfloat16)
        self.embed = torch.randn(vocab, self.hidden, generator=g, device=device).to(torch.bfloat16)
        self.w_qkv = [weight((hq + 2 * hk) * d, self.hidden) for _ in range(layers)]
        self.w_o = [weight(self.hidden, hq * d) for _ in range(layers)]
        self.w_gate_up = [weight(2 * inter, self.hidden) for _ in range(layers)]
        self.w_down = [weight(self.hidden, inter) for _ in range(layers)]
        self.packed = []
        for w in self.w_gate_up:
            self.packed.append(torch.empty_like(w))
            ppas.ppas_gateup_pack(w, self.packed[-1], self.hidden, inter)
        # the last projection: logits of a few units, as a trained model's
        self.w_out = (torch.randn(vocab, self.hidden, generator=g, device=device) * (2.0 / math.sqrt(self.hidden))).to(
            torch.bfloat16)
        f, self.rope_factor = ppas.ppas_rope_frequencies(ppas.PPAS_ROPE_PLAIN, d, 500000.0)
        self.inv_freq = torch.from_numpy(f).to(device)

    @staticmethod
    def norm(x):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(dim=-1, keepdim=True) + 1e-6)).to(torch.bfloat16)


class Answers:
    """The paged caches of one prompt and ``n`` answers of at most ``room`` tokens."""

    def __init__(self, model: Decoder, prompt, n: int, room: int, seed: int = 0, device="cuda"):
        geo = model.geo
        self.model, self.n, self.room, self.device = model, n, room, device
        self.prompt = torch.as_tensor(prompt, dtype=torch.int64, device=device)
        self.p_len = int(self.prompt.numel())
        if self.p_len < 1 or n < 1 or room < 1:
            raise ValueError("a prompt, an answer and a token at least")
        self.shared = self.p_len // PAGE                                  # pages that all answers read
        own = wl.blocks_for(self.p_len + room) - self.shared              # pages of one answer
        self.blocks = wl.blocks_for(self.p_len) + n * own
        order = np.random.default_rng(seed).permutation(self.blocks).astype(np.int32)
        n_prompt = wl.blocks_for(self.p_len)
        self.prompt_table = order[:n_prompt]
        self.table = np.concatenate([np.repeat(order[None, :self.shared], n, axis=0),
                                     order[n_prompt:].reshape(n, own)], axis=1)
        shape = (self.blocks, geo.n_kv_heads, PAGE, geo.head_dim)
        self.k = [torch.zeros(shape, dtype=torch.bfloat16, device=device) for _ in range(model.layers)]
        self.v = [torch.zeros(shape, dtype=torch.bfloat16, device=device) for _ in range(model.layers)]
        self.err = torch.zeros(1, dtype=torch.int32, device=device)
        self.ws = torch.empty(256, dtype=torch.uint8, device=device)

    def _workspace(self, size: int):
        if size > self.ws.numel():
            self.ws = torch.empty(size, dtype=torch.uint8, device=self.device)
        return self.ws

    def _layers(self, tokens, positions, slots, attention):
        """Hidden states of ``tokens`` after all layers; ``attention(layer, q, out)``."""
        m, geo = self.model, self.model.geo
        hq, hk, d = geo.n_q_heads, geo.n_kv_heads, geo.head_dim
        x = m.embed[tokens]
        t = x.shape[0]
        q = torch.empty((t, hq, d), dtype=torch.bfloat16, device=self.device)
        out = torch.empty_like(q)
        act = torch.empty((t, m.inter), dtype=torch.bfloat16, device=self.device)
        for i in range(m.layers):
            qkv = m.norm(x) @ m.w_qkv[i].T
            n = qkv.stride(0)
            ppas.ppas_rope_append(qkv, qkv[:, hq * d:], qkv[:, (hq + hk) * d:], n, n, n, positions, slots, t,
                                  m.inv_freq, d, False, m.rope_factor, q, self.k[i], self.v[i], self.blocks, hq, hk,
                                  d, self.err)
            attention(i, q, out)
            x = x + out.view(t, hq * d) @ m.w_o[i].T
            ppas.ppas_gateup_swiglu(m.norm(x), m.packed[i], act, t, m.hidden, m.inter, self.err)
            x = x + act @ m.w_down[i].T
        return m.norm(x)

    def prefill(self, chunk: int = 16384):
        """Computes the prompt; logits [1, vocab] (fp32) after its last token."""
        geo = self.model.geo
        table = torch.from_numpy(self.prompt_table.reshape(1, -1).copy()).to(self.device)
        last = None
        for a in range(0, self.p_len, chunk):
            b = min(self.p_len, a + chunk)
            pos = np.arange(a, b, dtype=np.int32)
            slots = self.prompt_table[pos // PAGE] * PAGE + pos % PAGE
            lens, ctx = np.array([b - a], np.int32), np.array([b], np.int32)
            size = ppas.ppas_attention_workspace_size(lens, ctx, geo.n_q_heads, geo.n_kv_heads)
            ws = self._workspace(size)

            def attention(i, q, out):
                ppas.ppas_attention_step(q, self.k[i], self.v[i], self.blocks, table, table.shape[1], lens, ctx,
                                         geo.n_q_heads, geo.n_kv_heads, geo.head_dim, geo.scale, out, False, ws, size,
                                         self.err)
            last = self._layers(self.prompt[a:b], torch.from_numpy(pos).to(self.device),
                                torch.from_numpy(slots.astype(np.int32)).to(self.device), attention)
        if self.p_len % PAGE:  # the page that is not full becomes each answer's own
            src = int(self.prompt_table[self.shared])
            dst = torch.from_numpy(self.table[:, self.shared].astype(np.int64)).to(self.device)
            for c in self.k + self.v:
                c[dst] = c[src].clone()
        return (last[-1:] @ self.model.w_out.T).float()

    def step(self, tokens, at: int):
        """One token of every answer, the ``at``-th after the prompt; logits [n, vocab] (fp32)."""
        geo = self.model.geo
        pos = self.p_len + at
        if not 0 <= at < self.room:
            raise ValueError("no room for this token")
        d_table = torch.from_numpy(self.table).to(self.device)
        slots = torch.from_numpy((self.table[:, pos // PAGE] * PAGE + pos % PAGE).astype(np.int32)).to(self.device)
        positions = torch.full((self.n,), pos, dtype=torch.int32, device=self.device)
        ctx = np.full(self.n, pos + 1, np.int32)
        rows, prefix = np.array([self.n], np.int32), np.array([self.shared * PAGE], np.int32)
        size = ppas.ppas_shared_attention_workspace_size(ctx, rows, prefix, geo.n_q_heads, geo.n_kv_heads)
        ws = self._workspace(size)

        def attention(i, q, out):
            ppas.ppas_shared_attention_step(q, self.k[i], self.v[i], self.blocks, d_table, d_table.shape[1], ctx, rows,
                                            prefix, geo.n_q_heads, geo.n_kv_heads, geo.head_dim, geo.scale, out, ws,
                                            size, self.err)
        return (self._layers(tokens.long(), positions, slots, attention) @ self.model.w_out.T).float()

    def check(self) -> None:
        if int(self.err.item()) != 0:
            raise RuntimeError(f"device error flag {int(self.err.item())}")


def draw(logits, rules: Rules, uniform, err=None):
    """(tokens, log-probabilities) of the rows of ``logits`` by ``rules`` and the given uniform numbers."""
    n, vocab = logits.shape
    dev = logits.device
    tokens = torch.empty(n, dtype=torch.int32, device=dev)
    logprobs = torch.empty(n, dtype=torch.float32, device=dev)
    ppas.ppas_sample_tokens(logits, logits.dtype == torch.bfloat16, logits.stride(0), n, vocab,
                            torch.full((n,), rules.temperature, device=dev),
                            torch.full((n,), rules.top_k, dtype=torch.int32, device=dev),
                            torch.full((n,), rules.top_p, device=dev), torch.full((n,), rules.min_p, device=dev),
                            uniform, tokens, logprobs, err)
    return tokens, logprobs


def generate(model: Decoder, prompt, n: int, length: int, rules: Rules = Rules(), seed: int = 0, on_step=None):
    """``n`` answers of ``length`` tokens to ``prompt``: (tokens [n, length], log-probabilities [n, length]).
    ``on_step(index, logits, uniform, tokens)`` sees every draw."""
    run = Answers(model, prompt, n, length, seed)
    g = torch.Generator(device=run.device)
    g.manual_seed(seed)
    logits = run.prefill().expand(n, -1).contiguous()
    tokens, logprobs = [], []
    for i in range(length):
        u = torch.rand(n, generator=g, device=run.device)
        t, lp = draw(logits, rules, u, run.err)
        if on_step is not None:
            on_step(i, logits, u, t)
        tokens.append(t)
        logprobs.append(lp)
        if i + 1 < length:
            logits = run.step(t, i)
    run.check()
    return torch.stack(tokens, dim=1), torch.stack(logprobs, dim=1)


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--prompt", type=int, default=25000, help="tokens of the prompt")
    ap.add_argument("--answers", type=int, default=32)
    ap.add_argument("--tokens", type=int, default=16, help="tokens of each answer")
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--temperature", type=float, default=0.8)
    ap.add_argument("--top-k", type=int, default=0)
    ap.add_argument("--top-p", type=float, default=0.95)
    ap.add_argument("--min-p", type=float, default=0.0)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    model = Decoder(layers=a.layers, seed=a.seed)
    prompt = np.random.default_rng(a.seed).integers(0, model.vocab, size=a.prompt)
    marks = []

    def mark(i, logits, uniform, tokens):
        marks.append(torch.cuda.Event(enable_timing=True))
        marks[-1].record()
    tokens, logprobs = generate(model, prompt, a.answers, a.tokens, Rules(a.temperature, a.top_k, a.top_p, a.min_p),
                                a.seed, mark)
    torch.cuda.synchronize()
    for r in range(min(4, a.answers)):
        print(f"answer {r}: tokens {tokens[r].tolist()}, log-probability {float(logprobs[r].sum()):.3f}")
    if len(marks) > 2:
        ms = marks[1].elapsed_time(marks[-1]) / (len(marks) - 2)
        print(f"{a.answers} answers over a prompt of {a.prompt}: {ms * 1000:.0f} us a token of all of them "
              f"({a.layers} layers)")


if __name__ == "__main__":
    main()
