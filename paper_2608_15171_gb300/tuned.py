"""Requests of differently fine-tuned models in one batch: one base decoder, a low-rank
adapter for each request, and the log probabilities, entropies and alternatives of
every token that is generated, or of a prompt's own tokens.

The planner (``ppas_plan_step``) composes every iteration of decodes and prefill
chunks as for any other load; all requests of an iteration, whatever their
adapters, then run through the layers together:

    qkv = norm(x) W_qkv            the shared projection, torch's
        + adapters                 ppas_adapter_add: each row its request's, q, k and v at once
    q, k = rotate(norm(heads))     ppas_norm_rope_append: normalised, rotated, appended
    x += attention W_o + adapters  ppas_attention_step, ppas_adapter_add
    x += gated MLP(norm(x))        ppas_gateup_swiglu, its last projection with adapters too

and the next tokens are drawn (``ppas_sample_tokens``) and looked up in the whole
distribution (``ppas_token_logprobs``).  The weights are random (there are no checkpoints
here).

    python -m paper_2608_15171_gb300.tuned --requests 12 --adapters 4 --tokens 8
"""
from __future__ import annotations

import argparse
import math
from dataclasses import dataclass, field
from typing import List

import numpy as np
import torch

from . import answers
from . import ppas
from . import workloads as wl


class TunedDecoder(answers.Decoder):
    """The decoder of ``answers`` with norms of query and key heads (which models of this
    geometry do not have; others do) and ``n_adapters`` adapters of ``rank``."""

    EPS = 1e-6

    def __init__(self, geo: wl.Geometry = wl.QWEN25_3B, layers: int = 2, vocab: int = 32000, inter: int = 4096,
                 n_adapters: int = 4, rank: int = 16, seed: int = 0, device="cuda"):
        super().__init__(geo, layers, vocab, inter, seed, device)
        g = torch.Generator(device=device)
        g.manual_seed(seed + 1)
        d, hq, hk = geo.head_dim, geo.n_q_heads, geo.n_kv_heads
        self.n_adapters, self.rank = n_adapters, rank

        def head_weight():
            return 1.0 + 0.2 * torch.randn(d, generator=g, device=device)
        self.q_norm = [head_weight() for _ in range(layers)]
        self.k_norm = [head_weight() for _ in range(layers)]

        def pair(hidden, slice_cols):
            a = torch.randn(n_adapters, len(slice_cols) * rank, hidden, generator=g, device=device) / math.sqrt(hidden)
            b = torch.randn(n_adapters, sum(slice_cols), rank, generator=g, device=device) / math.sqrt(rank)
            return a.to(torch.bfloat16), b.to(torch.bfloat16), np.array(slice_cols, np.int32)
        self.qkv_adapters = [pair(self.hidden, [hq * d, hk * d, hk * d]) for _ in range(layers)]
        self.o_adapters = [pair(hq * d, [self.hidden]) for _ in range(layers)]
        self.down_adapters = [pair(inter, [self.hidden]) for _ in range(layers)]
        self.scales = 0.5 + 0.5 * torch.rand(n_adapters, generator=g, device=device)


@dataclass
class Request:
    prompt: np.ndarray
    length: int                # tokens to generate
    adapter: int = -1          # -1: the base model
    tokens: List[int] = field(default_factory=list)
    logprobs: List[float] = field(default_factory=list)
    entropy: List[float] = field(default_factory=list)
    # the most likely tokens at every place, with their log probabilities
    alternatives: List[list] = field(default_factory=list)
    # log probabilities of the prompt's tokens from the second one on
    prompt_logprobs: List[float] = field(default_factory=list)


class Batch:
    """Runs requests to their ends, every planned iteration over all layers.  A request holds what
    was drawn for it, so it may be in one batch, once, and a batch runs once."""

    def __init__(self, model: TunedDecoder, requests, rules: answers.Rules = answers.Rules(), n_top: int = 5,
                 score_prompts: bool = False, mbt_hi: int = 16384, mbt_lo: int = 2048, seed: int = 0):
        self.model, self.requests, self.rules, self.n_top = model, list(requests), rules, n_top
        self.score_prompts, self.mbt_hi, self.mbt_lo = score_prompts, mbt_hi, mbt_lo
        geo, dev = model.geo, model.embed.device
        for r in self.requests:
            if len(r.prompt) < 1 or r.length < 1 or not -1 <= r.adapter < model.n_adapters:
                raise ValueError("a prompt, a token to generate and an adapter of the model, or -1")
            p = np.asarray(r.prompt)
            if p.ndim != 1 or not np.all((p >= 0) & (p < model.vocab) & (p.astype(np.int64) == p)):
                raise ValueError("a prompt of tokens of the vocabulary")
        self._check_fresh()
        self.blocks = sum(wl.blocks_for(len(r.prompt) + r.length) for r in self.requests) + 1
        shape = (self.blocks, geo.n_kv_heads, wl.PAGE_TOKENS, geo.head_dim)
        self.k = [torch.zeros(shape, dtype=torch.bfloat16, device=dev) for _ in range(model.layers)]
        self.v = [torch.zeros(shape, dtype=torch.bfloat16, device=dev) for _ in range(model.layers)]
        self.err = torch.zeros(1, dtype=torch.int32, device=dev)
        self.ws = torch.empty(256, dtype=torch.uint8, device=dev)
        self.generator = torch.Generator(device=dev)
        self.generator.manual_seed(seed)
        self.device, self.seed = dev, seed

    def _check_fresh(self) -> None:
        if len({id(r) for r in self.requests}) < len(self.requests) or \
                any(r.tokens or r.logprobs or r.entropy or r.alternatives or r.prompt_logprobs for r in self.requests):
            raise ValueError("a request may run once")

    def _adapt(self, x, y, q_lens, ids, adapters) -> None:
        """y += the requests' adapters of x, in place."""
        a, b, cols = adapters
        ppas.ppas_adapter_add(x, x.stride(0), y, y.stride(0), y, y.stride(0), q_lens, ids, a, b, self.model.scales,
                              self.model.n_adapters, x.shape[1], cols, self.model.rank, self.err)

    def _step(self, st: ppas.StepPlan):
        """Hidden states of one planned iteration's new tokens, after the last norm."""
        m, geo = self.model, self.model.geo
        hq, hk, d, t = geo.n_q_heads, geo.n_kv_heads, geo.head_dim, st.total_tokens
        ids = np.array([self.requests[i].adapter for i in st.req_idx], np.int32)
        tokens, positions = [], []
        for i, q, c in zip(st.req_idx, st.q_len, st.ctx_len):
            r = self.requests[i]
            tokens.append(np.concatenate([r.prompt, np.array(r.tokens, np.int64)])[c - q:c])
            positions.append(np.arange(c - q, c))
        pos = torch.from_numpy(np.concatenate(positions).astype(np.int32)).to(self.device)
        slots = torch.from_numpy(st.slot_mapping).to(self.device)
        tables = torch.from_numpy(st.block_table).to(self.device)
        size = ppas.ppas_attention_workspace_size(st.q_len, st.ctx_len, hq, hk)
        if size > self.ws.numel():
            self.ws = torch.empty(size, dtype=torch.uint8, device=self.device)
        x = m.embed[torch.from_numpy(np.concatenate(tokens).astype(np.int64)).to(self.device)]
        q = torch.empty((t, hq, d), dtype=torch.bfloat16, device=self.device)
        out = torch.empty_like(q)
        act = torch.empty((t, m.inter), dtype=torch.bfloat16, device=self.device)
        for i in range(m.layers):
            h = m.norm(x)
            qkv = h @ m.w_qkv[i].T
            self._adapt(h, qkv, st.q_len, ids, m.qkv_adapters[i])
            n = qkv.stride(0)
            ppas.ppas_norm_rope_append(qkv, qkv[:, hq * d:], qkv[:, (hq + hk) * d:], n, n, n, m.q_norm[i], m.k_norm[i],
                                       m.EPS, pos, slots, t, m.inv_freq, d, False, m.rope_factor, q, self.k[i],
                                       self.v[i], self.blocks, hq, hk, d, self.err)
            ppas.ppas_attention_step(q, self.k[i], self.v[i], self.blocks, tables, tables.shape[1], st.q_len,
                                     st.ctx_len, hq, hk, d, geo.scale, out, False, self.ws, size, self.err)
            o = out.view(t, hq * d) @ m.w_o[i].T
            self._adapt(out.view(t, hq * d), o, st.q_len, ids, m.o_adapters[i])
            x = x + o
            ppas.ppas_gateup_swiglu(m.norm(x), m.packed[i], act, t, m.hidden, m.inter, self.err)
            down = act @ m.w_down[i].T
            self._adapt(act, down, st.q_len, ids, m.down_adapters[i])
            x = x + down
        return m.norm(x)

    def _score(self, logits, tokens, n_top: int):
        """(log probabilities, entropies, top tokens, their log probabilities) of given tokens."""
        n, dev = logits.shape[0], self.device
        logprobs, entropy = (torch.empty(n, dtype=torch.float32, device=dev) for _ in range(2))
        top_tokens = torch.empty((n, n_top), dtype=torch.int32, device=dev)
        top_logprobs = torch.empty((n, n_top), dtype=torch.float32, device=dev)
        ppas.ppas_token_logprobs(logits, logits.dtype == torch.bfloat16, logits.stride(0), n, logits.shape[1], tokens,
                                 logprobs, entropy, n_top, top_tokens, top_logprobs, self.err)
        return logprobs, entropy, top_tokens, top_logprobs

    def run(self, on_logits=None, max_steps: int = 100000):
        """All requests to their ends; ``on_logits(request, place, row of logits)`` sees
        the logits behind every generated token.  RuntimeError if some have not ended
        after ``max_steps`` iterations."""
        self._check_fresh()
        sch = ppas.Scheduler(self.blocks, wl.page_permutation(self.blocks, self.seed), cap_rows=len(self.requests),
                             cap_blocks_per_seq=max(wl.blocks_for(len(r.prompt) + r.length) for r in self.requests),
                             cap_tokens=self.mbt_hi)
        sch.add_requests([(0, len(r.prompt), r.length) for r in self.requests])
        try:
            for now in range(max_steps):
                st = sch.plan(now, 2, self.mbt_hi, self.mbt_lo)
                if st.n_rows == 0:
                    break
                hidden = self._step(st)
                ends = np.cumsum(st.q_len)
                if self.score_prompts:
                    self._score_prompts(st, hidden, ends)
                # rows whose last new token has a successor to draw: decodes, and prompts that are complete
                rows = [j for j in range(st.n_rows) if st.ctx_len[j] >= len(self.requests[st.req_idx[j]].prompt)]
                if not rows:
                    continue
                last = torch.from_numpy((ends[rows] - 1).astype(np.int64)).to(self.device)
                logits = (hidden[last] @ self.model.w_out.T).float()
                uniform = torch.rand(len(rows), generator=self.generator, device=self.device)
                tokens, _ = answers.draw(logits, self.rules, uniform, self.err)
                scored = [x.tolist() for x in (tokens, *self._score(logits, tokens, self.n_top))]
                for place, j in enumerate(rows):
                    r = self.requests[st.req_idx[j]]
                    if on_logits is not None:
                        on_logits(int(st.req_idx[j]), len(r.tokens), logits[place])
                    token, logprob, entropy, top, top_logprobs = (x[place] for x in scored)
                    r.tokens.append(token)
                    r.logprobs.append(logprob)
                    r.entropy.append(entropy)
                    r.alternatives.append(list(zip(top, top_logprobs)))
        finally:
            sch.close()
        if int(self.err.item()) != 0:
            raise RuntimeError(f"device error flag {int(self.err.item())}")
        unfinished = [i for i, r in enumerate(self.requests) if len(r.tokens) < r.length]
        if unfinished:
            raise RuntimeError(f"requests {unfinished} are unfinished")
        return self.requests

    def _score_prompts(self, st, hidden, ends) -> None:
        """Log probabilities of prompt tokens behind this iteration's prefill chunks."""
        for j in range(st.n_rows):
            r = self.requests[st.req_idx[j]]
            a, b = int(st.ctx_len[j] - st.q_len[j]), min(int(st.ctx_len[j]), len(r.prompt) - 1)
            if a >= b:
                continue
            first = int(ends[j] - st.q_len[j])
            following = torch.from_numpy(np.asarray(r.prompt[a + 1:b + 1], np.int32)).to(self.device)
            logits = hidden[first:first + b - a] @ self.model.w_out.T
            r.prompt_logprobs += self._score(logits, following, 0)[0].tolist()


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--requests", type=int, default=12)
    ap.add_argument("--adapters", type=int, default=4)
    ap.add_argument("--rank", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=2000, help="tokens of the longest prompt")
    ap.add_argument("--tokens", type=int, default=8, help="tokens to generate for each request")
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--temperature", type=float, default=0.8)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args()
    model = TunedDecoder(layers=a.layers, n_adapters=a.adapters, rank=a.rank, seed=a.seed)
    rng = np.random.default_rng(a.seed)
    requests = [Request(rng.integers(0, model.vocab, size=int(rng.integers(1, a.prompt + 1))), a.tokens,
                        int(rng.integers(-1, a.adapters))) for _ in range(a.requests)]
    Batch(model, requests, answers.Rules(temperature=a.temperature), score_prompts=True, seed=a.seed).run()
    for i, r in enumerate(requests[:6]):
        mean = float(np.mean(r.prompt_logprobs)) if r.prompt_logprobs else float("nan")
        print(f"request {i} (adapter {r.adapter}, prompt {len(r.prompt)}, {mean:.2f} a prompt token): tokens {r.tokens}")
        print("    first token:", ", ".join(f"{t} {lp:.2f}" for t, lp in r.alternatives[0]),
              f"entropy {r.entropy[0]:.2f}")


if __name__ == "__main__":
    main()
