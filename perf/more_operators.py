"""The measured work of the operators that a step of requests with their own
fine-tuned adapters runs besides the mixed attention:

* ``norm_rope``: norms of the new tokens' queries and keys for each head, rotary
  positions, and the append of keys and values to the paged cache, in one pass
  (``ppas_norm_rope_append``).
* ``adapter``: the low-rank adapters of a step's requests beside a projection that
  all of them share (``ppas_adapter_add``).
* ``logprob``: log probabilities of given tokens, the entropy, and the most likely
  alternatives (``ppas_token_logprobs``).

With ``own`` false a pass computes them in elementary torch operations in 32
bits; with ``own`` true it makes the library's calls.

Attention geometries (16/2 and 32/8 heads of 128), MLP widths, 16-token pages, the
2k and 16k token budgets and the up to 30k positions are those of the repository's
workloads; ranks, vocabularies and counts of adapters are generic.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DIM = 128
EPS = 1e-6


# ------------------------------------------------------------------ the cases
def _norm_rope(name, tokens, hq, hk, rotary=128, interleaved=False, pos_hi=30000, padded=False, gain=1.0,
               lens_seed=0):
    return {"name": name, "kind": "norm_rope", "tokens": tokens, "hq": hq, "hk": hk, "rotary": rotary,
            "interleaved": interleaved, "pos_hi": pos_hi, "padded": padded, "gain": gain, "lens_seed": lens_seed}


def _adapter(name, decodes, chunks, hidden, slices, rank, adapters, none=0.0, lens_seed=0):
    return {"name": name, "kind": "adapter", "decodes": decodes, "chunks": chunks, "hidden": hidden,
            "slices": slices, "rank": rank, "adapters": adapters, "none": none, "lens_seed": lens_seed}


def _logprob(name, rows, vocab, n_top, bf16=False, spread=3.0, lens_seed=0):
    return {"name": name, "kind": "logprob", "rows": rows, "vocab": vocab, "n_top": n_top, "bf16": bf16,
            "spread": spread, "lens_seed": lens_seed}


def listed():
    return [
        # the one new token of a single user: the smallest call, bound by latency
        _norm_rope("norm_rope 1 token", 1, 16, 2, lens_seed=1),
        # a decode iteration of 64 requests, part of each head rotated in pairs of neighbours, long contexts
        _norm_rope("norm_rope 64 tokens, part of head", 64, 32, 8, rotary=64, interleaved=True, pos_hi=131072,
                   lens_seed=2),
        # an iteration under the 2k budget with 8 decodes, some rows only padding
        _norm_rope("norm_rope 2056 tokens", 2056, 16, 2, padded=True, lens_seed=3),
        # a prompt's first 16k chunk on the larger geometry, activations of uneven size
        _norm_rope("norm_rope 16384 tokens", 16384, 32, 8, gain=8.0, lens_seed=4),
        # one request's next token through the fused q/k/v projection
        _adapter("adapter 1 token", 1, "", 2048, "2048,256,256", 16, 4, lens_seed=5),
        # a decode iteration of 64 requests of many users on the larger geometry, one in eight without an adapter
        _adapter("adapter 64 decodes of 40", 64, "", 4096, "4096,1024,1024", 32, 40, none=0.125, lens_seed=6),
        # a step under the 2k budget: 8 decodes and chunks of other requests, odd lengths, the MLP's last projection
        _adapter("adapter 2k step", 8, "700,513,828,7", 11008, "2048", 16, 12, lens_seed=7),
        # a 16k step of long prompts and 4 decodes through the larger q/k/v projection, adapters of a high rank
        _adapter("adapter 16k step", 4, "9000,1380,6000", 4096, "4096,1024,1024", 64, 3, lens_seed=8),
        # one user's next token with its alternatives
        _logprob("logprob 1 x 152000", 1, 152000, 20, lens_seed=9),
        # a small vocabulary, odd in size, as the projection leaves it
        _logprob("logprob 64 x 32003 bf16", 64, 32003, 5, bf16=True, spread=2.0, lens_seed=10),
        # a large decode batch
        _logprob("logprob 256 x 152000", 256, 152000, 20, lens_seed=11),
        # scoring the tokens of a prompt's chunk, as the projection leaves the logits
        _logprob("logprob 4096 x 128000 bf16", 4096, 128000, 5, bf16=True, lens_seed=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["norm_rope", "adapter", "adapter", "logprob"])
    while True:
        if kind == "norm_rope":
            hq, hk = rng.choice([(16, 2), (16, 2), (32, 8), (32, 8), (8, 4), (8, 8)])
            c = _norm_rope("", _log_int(rng, 1, 16384), hq, hk, rotary=rng.choice([128, 128, 128, 96, 64, 32, 16]),
                           interleaved=rng.random() < 0.4, pos_hi=_log_int(rng, 16, 131072),
                           padded=rng.random() < 0.2, gain=rng.choice([0.1, 1.0, 1.0, 8.0]),
                           lens_seed=rng.randrange(1 << 20))
            fits = True
        elif kind == "adapter":
            decodes = rng.choice([0, _log_int(rng, 1, 128)])
            n = rng.choice([0, 0, 1, 2, 4, 9]) if decodes else rng.choice([1, 1, 2, 4, 9])
            chunks = [_log_int(rng, 2, 9000) for _ in range(n)]
            hidden, slices = rng.choice([(2048, "2048,256,256"), (2048, "2048"), (4096, "4096,1024,1024"),
                                         (4096, "4096"), (11008, "2048"), (14336, "4096"),
                                         (8 * _log_int(rng, 8, 600), str(8 * _log_int(rng, 8, 600)))])
            c = _adapter("", decodes, ",".join(map(str, chunks)), hidden, slices,
                         rng.choice([8, 16, 16, 24, 32, 64]), _log_int(rng, 1, 64), none=rng.choice([0.0, 0.0, 0.2]),
                         lens_seed=rng.randrange(1 << 20))
            w = work(c)
            fits = w["bytes"] <= 5.0e8 and w["flops"] <= 3.0e10 and w["flops"] > 0
        else:
            c = _logprob("", _log_int(rng, 1, 4096), _log_int(rng, 1000, 152000), rng.choice([0, 1, 5, 20, 32]),
                         bf16=rng.random() < 0.5, spread=rng.choice([0.5, 1.0, 2.0, 3.0, 5.0]),
                         lens_seed=rng.randrange(1 << 20))
            fits = work(c)["bytes"] <= 1.0e9
        del c["name"]
        if fits:
            return c


def _ints(text):
    return [int(x) for x in text.split(",")] if text else []


def _requests(case):
    """(new tokens of each request, adapter of each request, -1 without one); decodes first"""
    lens = [1] * case["decodes"] + _ints(case["chunks"])
    r = np.random.default_rng(case["lens_seed"])
    ids = r.integers(0, case["adapters"], size=len(lens))
    return np.array(lens, np.int32), np.where(r.random(len(lens)) < case["none"], -1, ids).astype(np.int32)


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, seed, scale=1.0):
    x = torch.randn(shape, generator=_generator(seed), device="cuda", dtype=torch.float32)
    return (x * scale).to(torch.bfloat16)


def prepare(case, seed):
    s = {"case": case, "err": torch.zeros(1, dtype=torch.int32, device="cuda")}
    rng = np.random.default_rng(seed)
    if case["kind"] == "norm_rope":
        t, hq, hk = case["tokens"], case["hq"], case["hk"]
        # the fused projection's rows: q, k and v of a token side by side
        s["qkv"] = _normal((t, (hq + 2 * hk) * DIM), seed * 16 + 1, case["gain"])
        s["q"], s["k"], s["v"] = s["qkv"].split([hq * DIM, hk * DIM, hk * DIM], dim=1)
        s["q_weight"], s["k_weight"] = (1.0 + 0.3 * torch.randn(DIM, generator=_generator(seed * 16 + n),
                                                                device="cuda") for n in (4, 5))
        s["blocks"] = -(-t // PAGE) + 8
        s["k_cache"] = _normal((s["blocks"], hk, PAGE, DIM), seed * 16 + 2)
        s["v_cache"] = _normal((s["blocks"], hk, PAGE, DIM), seed * 16 + 3)
        pos = np.arange(t) + int(rng.integers(0, max(1, case["pos_hi"] - t) + 1)) if t > 64 else \
            rng.integers(0, case["pos_hi"], size=t)
        order = rng.permutation(s["blocks"])
        slots = order[np.arange(t) // PAGE] * PAGE + np.arange(t) % PAGE
        if case["padded"]:
            slots[rng.random(t) < 0.05] = -1
        half = case["rotary"] // 2
        s["inv_freq"] = torch.tensor([500000.0 ** (-i / half) for i in range(half)], dtype=torch.float32).cuda()
        s["positions"] = torch.from_numpy(pos.astype(np.int32)).cuda()
        s["slots"] = torch.from_numpy(slots.astype(np.int32)).cuda()
        s["q_out"] = torch.empty((t, hq, DIM), dtype=torch.bfloat16, device="cuda")
        return s
    if case["kind"] == "adapter":
        hidden, rank, n = case["hidden"], case["rank"], case["adapters"]
        s["slices"] = np.array(_ints(case["slices"]), np.int32)
        cols = int(s["slices"].sum())
        s["lens"], s["ids"] = _requests(case)
        t = int(s["lens"].sum())
        s["x"] = _normal((t, hidden), seed * 16 + 1)
        s["y"] = _normal((t, cols), seed * 16 + 2)  # what the shared projection gave
        s["a"] = _normal((n, len(s["slices"]) * rank, hidden), seed * 16 + 3, hidden ** -0.5)
        s["b"] = _normal((n, cols, rank), seed * 16 + 4, 0.5 * rank ** -0.5)
        s["scales"] = torch.from_numpy(rng.choice([0.5, 1.0, 2.0], size=n).astype(np.float32)).cuda()
        s["out"] = torch.empty_like(s["y"])
        return s
    n, v = case["rows"], case["vocab"]
    g = _generator(seed * 16 + 1)
    x = torch.randn((n, v), generator=g, device="cuda")
    x *= case["spread"]
    # a few likely tokens stand out of the rest, and a few are banned
    likely = torch.randint(0, v, (n, 24), generator=g, device="cuda")
    x.scatter_add_(1, likely, torch.rand((n, 24), generator=g, device="cuda") * 3 * case["spread"])
    x.scatter_(1, torch.randint(0, v, (n, 16), generator=g, device="cuda"), -math.inf)
    s["logits"] = x.to(torch.bfloat16) if case["bf16"] else x
    # the given tokens: likely ones and any other
    any_token = torch.randint(0, v, (n,), generator=g, device="cuda")
    s["given"] = torch.where(torch.rand(n, generator=g, device="cuda") < 0.7, likely[:, 0], any_token).to(torch.int32)
    s["logprobs"] = torch.empty(n, dtype=torch.float32, device="cuda")
    s["entropy"] = torch.empty(n, dtype=torch.float32, device="cuda")
    s["top_tokens"] = torch.empty((n, case["n_top"]), dtype=torch.int32, device="cuda")
    s["top_logprobs"] = torch.empty((n, case["n_top"]), dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    if own:
        return _call(s)
    return {"norm_rope": _plain_norm_rope, "adapter": _plain_adapter, "logprob": _plain_logprob}[s["case"]["kind"]](s)


def _call(s):
    from paper_2608_15171_gb300 import ppas
    case = s["case"]
    if case["kind"] == "norm_rope":
        stride = s["qkv"].stride(0)
        ppas.ppas_norm_rope_append(s["q"], s["k"], s["v"], stride, stride, stride, s["q_weight"], s["k_weight"], EPS,
                                   s["positions"], s["slots"], case["tokens"], s["inv_freq"], case["rotary"],
                                   case["interleaved"], 1.0, s["q_out"], s["k_cache"], s["v_cache"], s["blocks"],
                                   case["hq"], case["hk"], DIM, s["err"])
        return {"q": s["q_out"], "k": s["k_cache"], "v": s["v_cache"], "err": s["err"]}
    if case["kind"] == "adapter":
        ppas.ppas_adapter_add(s["x"], case["hidden"], s["y"], s["y"].stride(0), s["out"], s["out"].stride(0),
                              s["lens"], s["ids"], s["a"], s["b"], s["scales"], case["adapters"], case["hidden"],
                              s["slices"], case["rank"], s["err"])
        return {"out": s["out"], "err": s["err"]}
    ppas.ppas_token_logprobs(s["logits"], case["bf16"], s["logits"].stride(0), case["rows"], case["vocab"],
                             s["given"], s["logprobs"], s["entropy"], case["n_top"], s["top_tokens"],
                             s["top_logprobs"], s["err"])
    return {"logprobs": s["logprobs"], "entropy": s["entropy"], "top_tokens": s["top_tokens"],
            "top_logprobs": s["top_logprobs"], "err": s["err"]}


# ------------------------------------------------------------------ the plain forms
def _plain_norm_rope(s):
    case = s["case"]
    t, half = case["tokens"], case["rotary"] // 2
    angle = s["positions"].double()[:, None, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def turn(x, heads, weight):
        x = x.reshape(t, heads, DIM).float()
        x = x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * weight
        a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if case["interleaved"] else \
            (x[..., :half], x[..., half:2 * half])
        u, w = a * cos - b * sin, b * cos + a * sin
        front = torch.stack([u, w], dim=-1).flatten(-2) if case["interleaved"] else torch.cat([u, w], dim=-1)
        return torch.cat([front, x[..., 2 * half:]], dim=-1).to(torch.bfloat16)

    keep = s["slots"] >= 0
    slots = s["slots"][keep].long()
    s["k_cache"][slots // PAGE, :, slots % PAGE] = turn(s["k"], case["hk"], s["k_weight"])[keep]
    s["v_cache"][slots // PAGE, :, slots % PAGE] = s["v"].reshape(t, case["hk"], DIM)[keep]
    return {"q": turn(s["q"], case["hq"], s["q_weight"]), "k": s["k_cache"], "v": s["v_cache"], "err": s["err"]}


def _plain_adapter(s):
    """Adapter by adapter: its rows gathered, both products, the sum."""
    rank = s["case"]["rank"]
    rows = np.repeat(s["ids"], s["lens"])
    scales = s["scales"]
    out = s["y"].clone()
    for n in sorted(set(int(i) for i in s["ids"]) - {-1}):
        mine = torch.from_numpy(np.flatnonzero(rows == n)).cuda()
        x, parts, at = s["x"][mine].float(), [], 0
        for j, cols in enumerate(s["slices"].tolist()):
            small = x @ s["a"][n, j * rank:(j + 1) * rank].float().T
            parts.append(small @ s["b"][n, at:at + cols].float().T)
            at += cols
        out[mine] = (s["y"][mine].float() + scales[n] * torch.cat(parts, dim=1)).to(torch.bfloat16)
    return {"out": out, "err": s["err"]}


def _plain_logprob(s):
    case = s["case"]
    x = s["logits"].float()
    top = x.amax(dim=1, keepdim=True)
    z = x - top
    e = torch.exp(z)
    total = e.sum(dim=1, keepdim=True, dtype=torch.float64)
    log_total = torch.log(total)
    spread = torch.where(e > 0, z * e, 0.0).sum(dim=1, keepdim=True, dtype=torch.float64)
    entropy = (log_total - spread / total).float()[:, 0]
    logprobs = (z.gather(1, s["given"].long()[:, None]) - log_total).float()[:, 0]
    # the largest logits, the lowest index of equal ones: both in one whole number
    bits = (x + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 20) - torch.arange(case["vocab"], device="cuda")
    place = torch.topk(key, case["n_top"], dim=1, sorted=True).indices
    found = z.gather(1, place)
    return {"logprobs": logprobs, "entropy": entropy,
            "top_tokens": torch.where(found > -math.inf, place, -1).to(torch.int32),
            "top_logprobs": (found - log_total).float(), "err": s["err"]}


def work(case):
    if case["kind"] == "norm_rope":
        t, hq, hk = case["tokens"], case["hq"], case["hk"]
        return {"bytes": t * (hq + 2 * hk) * DIM * 4 + 8 * t + 2 * case["rotary"] + 8 * DIM,
                "flops": t * (hq + hk) * (4 * DIM + 3 * case["rotary"])}
    if case["kind"] == "adapter":
        lens, ids = _requests(case)
        slices = _ints(case["slices"])
        cols, wide = sum(slices), len(slices) * case["rank"]
        rows, used = int(lens[ids >= 0].sum()), len(set(ids.tolist()) - {-1})
        each = wide * case["hidden"] + cols * case["rank"]
        return {"bytes": 2 * (rows * case["hidden"] + 2 * int(lens.sum()) * cols + used * each) + 4 * used,
                "flops": 2 * rows * each}
    n, v = case["rows"], case["vocab"]
    return {"bytes": n * v * (2 if case["bf16"] else 4) + n * (12 + 8 * case["n_top"]), "flops": 4 * n * v}


# ------------------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm_rope": _exact_norm_rope, "adapter": _exact_adapter, "logprob": _exact_logprob}[case["kind"]](s)


def _exact_norm_rope(s):
    case = s["case"]
    t, r = case["tokens"], case["rotary"]
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()[None, :]
    turn = torch.polar(torch.ones_like(angle), angle)[:, None, :]

    def turned(x, heads, weight):
        y = x.contiguous().double().view(t, heads, DIM)
        y = y / torch.sqrt(y.square().sum(dim=-1, keepdim=True) / DIM + EPS) * weight.double()
        if case["interleaved"]:
            pairs = torch.view_as_complex(y[..., :r].reshape(t, heads, r // 2, 2).contiguous())
            y[..., :r] = torch.view_as_real(pairs * turn).reshape(t, heads, r)
        else:
            pairs = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous()) * turn
            y[..., :r // 2], y[..., r // 2:r] = pairs.real, pairs.imag
        return y

    got = {"q": turned(s["q"], case["hq"], s["q_weight"]), "err": None}
    for name, rows in (("k", turned(s["k"], case["hk"], s["k_weight"])),
                       ("v", s["v"].double().reshape(t, case["hk"], DIM))):
        flat = s[name + "_cache"].double().transpose(1, 2).reshape(-1, case["hk"], DIM)
        flat[s["slots"][s["slots"] >= 0].long()] = rows[s["slots"] >= 0]
        got[name] = flat.view(s["blocks"], PAGE, case["hk"], DIM).transpose(1, 2)
    return got


def _exact_adapter(s):
    """Request by request."""
    case = s["case"]
    of_slice = torch.from_numpy(np.repeat(np.arange(len(s["slices"])), s["slices"])).cuda()
    out = s["y"].double()
    at = 0
    for n, adapter in zip(s["lens"].tolist(), s["ids"].tolist()):
        if adapter >= 0:
            small = s["x"][at:at + n].double() @ s["a"][adapter].double().T
            small = small.view(n, len(s["slices"]), case["rank"])
            for j in range(len(s["slices"])):
                b = s["b"][adapter][of_slice == j].double()
                out[at:at + n, of_slice == j] += s["scales"][adapter].double() * (small[:, j] @ b.T)
        at += n
    return {"out": out, "err": None}


def _exact_logprob(s):
    """A few rows at a time: log probabilities in 64 bits, sorted."""
    case = s["case"]
    n, k = case["rows"], case["n_top"]
    got = {"logprobs": torch.empty(n, dtype=torch.float64, device="cuda"),
           "entropy": torch.empty(n, dtype=torch.float64, device="cuda"),
           "top_tokens": torch.empty((n, k), dtype=torch.int64, device="cuda"),
           "top_logprobs": torch.empty((n, k), dtype=torch.float64, device="cuda"), "err": None}
    step = max(1, (1 << 23) // case["vocab"])
    for a in range(0, n, step):
        x = s["logits"][a:a + step].double()
        lp = x - torch.logsumexp(x, dim=1, keepdim=True)
        rows = torch.arange(lp.shape[0], device="cuda")
        got["logprobs"][a:a + step] = lp[rows, s["given"][a:a + step].long()]
        got["entropy"][a:a + step] = -torch.special.xlogy(torch.exp(lp), torch.exp(lp)).sum(dim=1)
        if k:
            value, index = torch.sort(lp, dim=1, descending=True, stable=True)
            got["top_logprobs"][a:a + step] = value[:, :k]
            got["top_tokens"][a:a + step] = torch.where(value[:, :k] > -math.inf, index[:, :k], -1)
    return got
