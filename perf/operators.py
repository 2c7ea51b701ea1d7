"""The measured work of the operators that a decode iteration of many answers to
one prompt runs besides the ordinary step:

* ``rope``: rotary positions of the new tokens' queries and keys, and the append
  of their keys and values to the paged cache (``ppas_rope_append``).
* ``shared``: attention of single-token rows in groups whose rows share a long
  prefix (``ppas_shared_attention_step``).
* ``sample``: the next tokens from the logits with temperature, top-k, top-p and
  min-p, from given uniform numbers (``ppas_sample_tokens``).

With ``own`` false a pass computes them in elementary torch operations in 32
bits; with ``own`` true it makes the library's calls.

Attention geometries (16/2 and 32/8 heads of 128), 16-token pages in random order,
the 2k and 16k token budgets and the 2k-30k contexts are those of the repository's
workloads; vocabularies and counts of answers are generic.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
DIM = 128
UNIT = float(1 << 40)  # sampling weights are whole multiples of 2^-40 of the largest


# ------------------------------------------------------------------ the cases
def _rope(name, tokens, hq, hk, rotary=128, interleaved=False, pos_hi=30000, scaled=False, padded=False, lens_seed=0):
    return {"name": name, "kind": "rope", "tokens": tokens, "hq": hq, "hk": hk, "rotary": rotary,
            "interleaved": interleaved, "pos_hi": pos_hi, "scaled": scaled, "padded": padded, "lens_seed": lens_seed}


def _shared(name, hq, hk, rows, prefixes, own_lo, own_hi, gain=1.0, lens_seed=0):
    return {"name": name, "kind": "shared", "hq": hq, "hk": hk, "rows": rows, "prefixes": prefixes, "own_lo": own_lo,
            "own_hi": own_hi, "gain": gain, "lens_seed": lens_seed}


def _sample(name, rows, vocab, bf16=False, spread=3.0, rules="mixed", lens_seed=0):
    return {"name": name, "kind": "sample", "rows": rows, "vocab": vocab, "bf16": bf16, "spread": spread,
            "rules": rules, "lens_seed": lens_seed}


def listed():
    return [
        # the one new token of a single user: the smallest call, bound by latency
        _rope("rope 1 token", 1, 16, 2, lens_seed=1),
        # a decode iteration of 64 answers, half of each head rotated in pairs of neighbours, long-context frequencies
        _rope("rope 64 tokens, part of head", 64, 32, 8, rotary=64, interleaved=True, pos_hi=131072, scaled=True,
              lens_seed=2),
        # an iteration under the 2k budget with 8 decodes, some rows only padding
        _rope("rope 2056 tokens", 2056, 16, 2, padded=True, lens_seed=3),
        # a prompt's first 16k chunk on the larger geometry
        _rope("rope 16384 tokens", 16384, 32, 8, scaled=True, lens_seed=4),
        # four answers to a short prompt, just begun
        _shared("shared 4 x 2k", 16, 2, "4", "2048", 1, 64, lens_seed=5),
        # 32 answers to a 25k prompt
        _shared("shared 32 x 25k", 16, 2, "32", "24992", 17, 500, lens_seed=6),
        # the same on the larger geometry, 64 answers to 30k tokens, up to 1000 tokens into them
        _shared("shared 64 x 30k", 32, 8, "64", "30000", 1, 1000, lens_seed=7),
        # several prompts at once, one of them with a single answer and one without a prefix
        _shared("shared 5 groups", 16, 2, "9,33,1,21,6", "4096,25008,9984,512,0", 1, 300, lens_seed=8),
        # one user's next token
        _sample("sample 1 x 152000", 1, 152000, rules="nucleus", lens_seed=9),
        # answers of several users, each with its own rules; logits as the projection leaves them
        _sample("sample 32 x 128000 bf16", 32, 128000, bf16=True, lens_seed=10),
        # a small vocabulary, odd in size
        _sample("sample 64 x 32003", 64, 32003, spread=2.0, lens_seed=11),
        # the largest batch
        _sample("sample 256 x 152000", 256, 152000, lens_seed=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["rope", "shared", "shared", "sample"])
    while True:
        if kind == "rope":
            hq, hk = rng.choice([(16, 2), (16, 2), (32, 8), (32, 8), (8, 4), (8, 8)])
            c = _rope("", _log_int(rng, 1, 16384), hq, hk, rotary=rng.choice([128, 128, 128, 96, 64, 32, 16]),
                      interleaved=rng.random() < 0.4, pos_hi=_log_int(rng, 16, 131072), scaled=rng.random() < 0.5,
                      padded=rng.random() < 0.2, lens_seed=rng.randrange(1 << 20))
            fits = True
        elif kind == "shared":
            hq, hk = rng.choice([(16, 2), (16, 2), (32, 8), (32, 8), (8, 4), (8, 8)])
            n = rng.choice([1, 1, 1, 2, 3, 5])
            rows = [_log_int(rng, 1, 64) for _ in range(n)]
            prefixes = [0 if rng.random() < 0.1 else PAGE * _log_int(rng, 1, 1875) for _ in range(n)]
            lo = rng.choice([0, 1, 1, 16]) if min(prefixes) > 0 else 1
            c = _shared("", hq, hk, ",".join(map(str, rows)), ",".join(map(str, prefixes)), lo,
                        lo + _log_int(rng, 1, 1000), gain=rng.choice([1.0, 1.0, 2.0, 4.0]),
                        lens_seed=rng.randrange(1 << 20))
            w = work(c)
            fits = (sum(rows) * (max(prefixes) + c["own_hi"]) * hk <= 64 * 31000 * 8 and w["bytes"] <= 2.6e8 and
                    w["flops"] <= 3.2e10)
        else:
            c = _sample("", _log_int(rng, 1, 256), _log_int(rng, 1000, 152000), bf16=rng.random() < 0.4,
                        spread=rng.choice([0.5, 1.0, 2.0, 3.0, 5.0]),
                        rules=rng.choice(["mixed", "mixed", "nucleus", "top-k", "plain"]),
                        lens_seed=rng.randrange(1 << 20))
            fits = True
        del c["name"]
        if fits:
            return c


def _ints(text):
    return [int(x) for x in text.split(",")]


def _lens(case):
    """(rows of each group, prefix of each group, context of each row)"""
    rows, prefixes = _ints(case["rows"]), _ints(case["prefixes"])
    r = np.random.default_rng(case["lens_seed"])
    ctx = [p + int(x) for n, p in zip(rows, prefixes)
           for x in r.integers(case["own_lo"], case["own_hi"] + 1, size=n)]
    return rows, prefixes, ctx


# ------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(shape, seed):
    return torch.randn(shape, generator=_generator(seed), device="cuda", dtype=torch.float32).to(torch.bfloat16)


def _frequencies(case):
    """(inverse frequencies, factor on cosine and sine): base 500000, and where
    scaled the long wavelengths stretched by 8, with a ramp between 1/4 and 1 of 8192 positions."""
    half = case["rotary"] // 2
    f = [500000.0 ** (-i / half) for i in range(half)]
    if case["scaled"]:
        ratio = [8192 * x / (2 * math.pi) for x in f]
        ramp = [min(1.0, max(0.0, (x - 1.0) / 3.0)) for x in ratio]
        f = [x * a + x / 8 * (1 - a) for x, a in zip(f, ramp)]
    return f, 0.1 * math.log(8.0) + 1.0 if case["scaled"] else 1.0


def prepare(case, seed):
    s = {"case": case, "err": torch.zeros(1, dtype=torch.int32, device="cuda")}
    rng = np.random.default_rng(seed)
    if case["kind"] == "rope":
        t, hq, hk = case["tokens"], case["hq"], case["hk"]
        # the fused projection's rows: q, k and v of a token side by side
        s["qkv"] = _normal((t, (hq + 2 * hk) * DIM), seed * 16 + 1)
        s["q"], s["k"], s["v"] = s["qkv"].split([hq * DIM, hk * DIM, hk * DIM], dim=1)
        s["blocks"] = -(-t // PAGE) + 8
        s["k_cache"] = _normal((s["blocks"], hk, PAGE, DIM), seed * 16 + 2)
        s["v_cache"] = _normal((s["blocks"], hk, PAGE, DIM), seed * 16 + 3)
        pos = np.arange(t) + int(rng.integers(0, max(1, case["pos_hi"] - t) + 1)) if t > 64 else \
            rng.integers(0, case["pos_hi"], size=t)
        order = rng.permutation(s["blocks"])
        slots = order[np.arange(t) // PAGE] * PAGE + np.arange(t) % PAGE
        if case["padded"]:
            slots[rng.random(t) < 0.05] = -1
        f, s["factor"] = _frequencies(case)
        s["inv_freq"] = torch.tensor(f, dtype=torch.float32).cuda()
        s["positions"] = torch.from_numpy(pos.astype(np.int32)).cuda()
        s["slots"] = torch.from_numpy(slots.astype(np.int32)).cuda()
        s["q_out"] = torch.empty((t, hq, DIM), dtype=torch.bfloat16, device="cuda")
        return s
    if case["kind"] == "shared":
        hq, hk = case["hq"], case["hk"]
        rows, prefixes, ctx = _lens(case)
        group = np.repeat(np.arange(len(rows)), rows)
        first = [p // PAGE for p in prefixes]
        mine = [-(-c // PAGE) - first[g] for c, g in zip(ctx, group)]
        s["blocks"] = sum(first) + sum(mine) + 8
        order = rng.permutation(s["blocks"]).astype(np.int32)
        table = np.full((len(ctx), max(first[g] + m for g, m in zip(group, mine))), -1, np.int32)
        ends = np.cumsum(first)
        at = int(ends[-1])
        for r, (g, m) in enumerate(zip(group, mine)):
            table[r, :first[g]] = order[ends[g] - first[g]:ends[g]]
            table[r, first[g]:first[g] + m] = order[at:at + m]
            at += m
        s["rows"], s["prefixes"] = np.array(rows, np.int32), np.array(prefixes, np.int32)
        s["ctx_lens"], s["table_host"], s["width"] = np.array(ctx, np.int32), table, table.shape[1]
        s["table"], s["ctx"] = torch.from_numpy(table).cuda(), torch.from_numpy(s["ctx_lens"]).cuda()
        s["q"] = _normal((len(ctx), hq, DIM), seed * 16 + 1) * case["gain"]
        s["k_cache"] = _normal((s["blocks"], hk, PAGE, DIM), seed * 16 + 2)
        s["v_cache"] = _normal((s["blocks"], hk, PAGE, DIM), seed * 16 + 3)
        s["out"] = torch.empty((len(ctx), hq, DIM), dtype=torch.bfloat16, device="cuda")
        return s
    n, v = case["rows"], case["vocab"]
    g = _generator(seed * 16 + 1)
    x = torch.randn((n, v), generator=g, device="cuda") * case["spread"]
    # a few likely tokens stand out of the rest, and a few are banned
    likely = torch.randint(0, v, (n, 24), generator=g, device="cuda")
    x.scatter_add_(1, likely, torch.rand((n, 24), generator=g, device="cuda") * 3 * case["spread"])
    x.scatter_(1, torch.randint(0, v, (n, 16), generator=g, device="cuda"), -math.inf)
    s["logits"] = x.to(torch.bfloat16) if case["bf16"] else x
    r = np.random.default_rng(case["lens_seed"])
    pick = {"plain": [(1.0, 0, 1.0, 0.0)], "nucleus": [(0.8, 0, 0.95, 0.0)], "top-k": [(0.7, 50, 1.0, 0.0)],
            "mixed": [(0.8, 0, 0.95, 0.0), (1.0, 0, 1.0, 0.0), (0.7, 50, 1.0, 0.0), (0.0, 0, 1.0, 0.0),
                      (1.0, 0, 1.0, 0.05), (0.6, 40, 0.9, 0.02), (1.3, 1000, 0.98, 0.0), (1.0, 0, 0.5, 0.0)]}
    rules = pick[case["rules"]]
    of = r.integers(0, len(rules), size=n)
    s["temperature"], s["top_p"], s["min_p"] = (
        torch.tensor([rules[i][j] for i in of], dtype=torch.float32).cuda() for j in (0, 2, 3))
    s["top_k"] = torch.tensor([rules[i][1] for i in of], dtype=torch.int32).cuda()
    s["uniform"] = torch.rand(n, generator=g, device="cuda")
    s["tokens"] = torch.empty(n, dtype=torch.int32, device="cuda")
    s["logprobs"] = torch.empty(n, dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    if own:
        return _call(s)
    return {"rope": _plain_rope, "shared": _plain_shared, "sample": _plain_sample}[s["case"]["kind"]](s)


def _call(s):
    from paper_2608_15171_gb300 import ppas
    case = s["case"]
    if case["kind"] == "rope":
        stride = s["qkv"].stride(0)
        ppas.ppas_rope_append(s["q"], s["k"], s["v"], stride, stride, stride, s["positions"], s["slots"],
                              case["tokens"], s["inv_freq"], case["rotary"], case["interleaved"], s["factor"],
                              s["q_out"], s["k_cache"], s["v_cache"], s["blocks"], case["hq"], case["hk"], DIM,
                              s["err"])
        return {"q": s["q_out"], "k": s["k_cache"], "v": s["v_cache"], "err": s["err"]}
    if case["kind"] == "shared":
        if "ws" not in s:  # one workspace for all the layers of an iteration
            s["ws_bytes"] = ppas.ppas_shared_attention_workspace_size(s["ctx_lens"], s["rows"], s["prefixes"],
                                                                      case["hq"], case["hk"])
            s["ws"] = torch.empty(max(s["ws_bytes"], 256), dtype=torch.uint8, device="cuda")
        ppas.ppas_shared_attention_step(s["q"], s["k_cache"], s["v_cache"], s["blocks"], s["table"], s["width"],
                                        s["ctx_lens"], s["rows"], s["prefixes"], case["hq"], case["hk"], DIM,
                                        DIM ** -0.5, s["out"], s["ws"], s["ws_bytes"], s["err"])
        return {"out": s["out"], "err": s["err"]}
    ppas.ppas_sample_tokens(s["logits"], case["bf16"], s["logits"].stride(0), case["rows"], case["vocab"],
                            s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["uniform"], s["tokens"],
                            s["logprobs"], s["err"])
    return {"tokens": s["tokens"], "logprobs": s["logprobs"], "err": s["err"]}


# ------------------------------------------------------------------ the plain forms
def _plain_rope(s):
    case = s["case"]
    t, half = case["tokens"], case["rotary"] // 2
    angle = s["positions"].float()[:, None, None] * s["inv_freq"]
    cos, sin = torch.cos(angle) * s["factor"], torch.sin(angle) * s["factor"]

    def turn(x, heads):
        x = x.reshape(t, heads, DIM).float()
        a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if case["interleaved"] else \
            (x[..., :half], x[..., half:2 * half])
        u, w = a * cos - b * sin, b * cos + a * sin
        front = torch.stack([u, w], dim=-1).flatten(-2) if case["interleaved"] else torch.cat([u, w], dim=-1)
        return torch.cat([front, x[..., 2 * half:]], dim=-1).to(torch.bfloat16)

    keep = s["slots"] >= 0
    slots = s["slots"][keep].long()
    s["k_cache"][slots // PAGE, :, slots % PAGE] = turn(s["k"], case["hk"])[keep]
    s["v_cache"][slots // PAGE, :, slots % PAGE] = s["v"].reshape(t, case["hk"], DIM)[keep]
    return {"q": turn(s["q"], case["hq"]), "k": s["k_cache"], "v": s["v_cache"], "err": s["err"]}


def _plain_shared(s):
    case = s["case"]
    hq, hk = case["hq"], case["hk"]
    n, width = s["table"].shape
    pages = s["table"].clamp(min=0).long()

    def dense(cache):
        return cache[pages].permute(0, 2, 1, 3, 4).reshape(n, hk, width * PAGE, DIM).float()

    w = (s["q"].float().view(n, hk, hq // hk, DIM) @ dense(s["k_cache"]).transpose(-1, -2)) * DIM ** -0.5
    past = torch.arange(width * PAGE, device="cuda") >= s["ctx"][:, None]
    w.masked_fill_(past[:, None, None, :], -math.inf)
    w = torch.exp(w - w.amax(dim=-1, keepdim=True))
    out = (w @ dense(s["v_cache"])) / w.sum(dim=-1, keepdim=True)
    return {"out": out.reshape(n, hq, DIM).to(torch.bfloat16), "err": s["err"]}


def _plain_sample(s):
    n, v = s["logits"].shape
    x = s["logits"].float() + 0.0  # a negative zero is a zero
    x = torch.where(torch.isnan(x), -math.inf, x)
    top = x.amax(dim=1, keepdim=True)
    hot = s["temperature"] > 0
    z = (x - top) * (1.0 / torch.where(hot, s["temperature"], 1.0))[:, None]
    z = torch.where(x == top, 0.0, z)
    w = (torch.where(x == -math.inf, 0.0, torch.exp(z)).double() * UNIT).to(torch.int64)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    cum = torch.cumsum(w.gather(1, order), dim=1)

    def at(count):
        return cum.gather(1, (count - 1)[:, None])[:, 0]

    k = s["top_k"].long()
    count = torch.where((k > 0) & (k < v), k, v)
    target = torch.ceil(s["top_p"].double() * at(count).double()).to(torch.int64)
    nucleus = 1 + (cum < target[:, None]).sum(dim=1)
    above = ((z >= torch.log(s["min_p"])[:, None]) & (x > -math.inf)).sum(dim=1).clamp(min=1)
    count = torch.where(s["top_p"] < 1, torch.minimum(count, nucleus), count)
    count = torch.where(s["min_p"] > 0, torch.minimum(count, above), count)
    count = torch.where(hot, count, 1)
    total = at(count)
    t = torch.minimum((s["uniform"].double() * total.double()).to(torch.int64), total - 1).clamp(min=0)
    place = (cum <= t[:, None]).sum(dim=1).clamp(max=v - 1)
    token = order.gather(1, place[:, None])
    mass = w.gather(1, token)[:, 0]
    rest = torch.log1p(-((total - mass).float() / total.float()))
    logprob = torch.where(2 * mass > total, rest, torch.log(mass.float() / total.float()))
    some = total > 0
    return {"tokens": torch.where(some, token[:, 0], -1).to(torch.int32),
            "logprobs": torch.where(some, logprob, -math.inf), "err": s["err"]}


def work(case):
    if case["kind"] == "rope":
        t, hq, hk = case["tokens"], case["hq"], case["hk"]
        return {"bytes": t * (hq + 2 * hk) * DIM * 4 + 8 * t + 2 * case["rotary"],
                "flops": 3 * t * (hq + hk) * case["rotary"]}
    if case["kind"] == "shared":
        rows, prefixes, ctx = _lens(case)
        hq, hk = case["hq"], case["hk"]
        keys = sum(prefixes) + sum(ctx) - sum(n * p for n, p in zip(rows, prefixes))
        return {"bytes": keys * hk * DIM * 4 + len(ctx) * hq * DIM * 4,
                "flops": 4 * DIM * hq * sum(ctx)}
    n, v = case["rows"], case["vocab"]
    return {"bytes": n * v * (2 if case["bf16"] else 4) + 28 * n, "flops": 4 * n * v}


# ------------------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "shared": _exact_shared, "sample": _exact_sample}[case["kind"]](s)


def _exact_rope(s):
    case = s["case"]
    t, r = case["tokens"], case["rotary"]
    turn = torch.polar(torch.full((1, 1), s["factor"], dtype=torch.float64, device="cuda"),
                       s["positions"].double()[:, None] * s["inv_freq"].double()[None, :])[:, None, :]

    def rotated(x, heads):
        y = x.double().view(t, heads, DIM).clone()
        if case["interleaved"]:
            pairs = torch.view_as_complex(y[..., :r].reshape(t, heads, r // 2, 2).contiguous())
            y[..., :r] = torch.view_as_real(pairs * turn).reshape(t, heads, r)
        else:
            pairs = torch.complex(y[..., :r // 2].contiguous(), y[..., r // 2:r].contiguous()) * turn
            y[..., :r // 2], y[..., r // 2:r] = pairs.real, pairs.imag
        return y

    got = {"q": rotated(s["q"].contiguous(), case["hq"]), "err": None}
    for name, rows in (("k", rotated(s["k"].contiguous(), case["hk"])),
                       ("v", s["v"].double().reshape(t, case["hk"], DIM))):
        flat = s[name + "_cache"].double().transpose(1, 2).reshape(-1, case["hk"], DIM)
        flat[s["slots"][s["slots"] >= 0].long()] = rows[s["slots"] >= 0]
        got[name] = flat.view(s["blocks"], PAGE, case["hk"], DIM).transpose(1, 2)
    return got


def _exact_shared(s):
    case = s["case"]
    hq, hk = case["hq"], case["hk"]
    out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    for r, c in enumerate(s["ctx_lens"].tolist()):
        pages = torch.from_numpy(s["table_host"][r, :-(-c // PAGE)]).cuda().long()
        k, v = (s[n][pages].transpose(0, 1).reshape(hk, -1, DIM)[:, :c].double() for n in ("k_cache", "v_cache"))
        w = torch.softmax((s["q"][r].double().view(hk, hq // hk, DIM) @ k.transpose(1, 2)) / math.sqrt(DIM), dim=-1)
        out[r] = (w @ v).reshape(hq, DIM)
    return {"out": out, "err": None}


def _exact_sample(s):
    """One row after another, from the definition: probabilities in 64 bits,
    sorted, cut, renormalised, and the draw by inversion.  (A draw at the edge of
    two tokens may go either way by rounding: no value is given for the tokens.)"""
    logprobs = []
    temperature, top_k, top_p, min_p, uniform = (
        s[n].tolist() for n in ("temperature", "top_k", "top_p", "min_p", "uniform"))
    for r in range(s["case"]["rows"]):
        if temperature[r] <= 0:
            logprobs.append(0.0)
            continue
        x = s["logits"][r].double()
        p = torch.sort(torch.softmax(x / temperature[r], dim=0), descending=True).values
        if 0 < top_k[r] < p.numel():
            p = p[:top_k[r]]
        p = p / p.sum()
        if top_p[r] < 1:
            p = p[:int((torch.cumsum(p, dim=0) < top_p[r]).sum()) + 1]
        if min_p[r] > 0:
            p = p[p >= min_p[r] * p[0]]
        p = p / p.sum()
        at = min(int((torch.cumsum(p, dim=0) <= uniform[r]).sum()), p.numel() - 1)
        logprobs.append(math.log(float(p[at])))
    return {"tokens": None, "logprobs": torch.tensor(logprobs, dtype=torch.float64), "err": None}
