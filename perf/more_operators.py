"""Cases of the decoder's attention operators: inputs, plain forms, exact values.

Operators (``op``):
  qk      norms of queries and keys for each head, with the position rotation; ``append``: keys and values go into the
          4-bit cache in the same call and are read back
  store   keys and values into the 4-bit cache, and read back
  decode  attention of each sequence's last tokens over the 4-bit cache
  prompt  causal attention over whole prompts, packed one after another
Rows of the cache are returned as the values they stand for, in 16 bits.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
VALUES = {"f32": torch.bfloat16, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


def listed():
    return [
        # one decoded token between its products: queries out, its key and value into the cache; latency
        {"name": "qk one token", "op": "qk", "tokens": 1, "heads": 32, "kv": 8, "dim": 128, "rot": 128, "interleaved": False,
         "norm": True, "dtype": "bf16", "append": True, "page": 64},
        # a long prompt's queries and keys: bandwidth
        {"name": "qk prompt", "op": "qk", "tokens": 8192, "heads": 32, "kv": 8, "dim": 128, "rot": 128, "interleaved": False,
         "norm": True, "dtype": "bf16", "append": False},
        # a small model in 32 bits that rotates a part of each head, in adjacent pairs
        {"name": "qk odd f32", "op": "qk", "tokens": 777, "heads": 14, "kv": 2, "dim": 64, "rot": 32, "interleaved": True,
         "norm": True, "dtype": "f32", "append": False},
        # a batch of decoded tokens' keys and values
        {"name": "store batch", "op": "store", "tokens": 100, "kv": 8, "dim": 128, "dtype": "f16", "page": 16},
        # a long prompt's
        {"name": "store prompt", "op": "store", "tokens": 16384, "kv": 8, "dim": 128, "dtype": "bf16", "page": 64},
        # one token of one short conversation: latency
        {"name": "decode one", "op": "decode", "seqs": 1, "longest": 1000, "queries": 1, "heads": 32, "kv": 8, "dim": 128,
         "dtype": "bf16", "page": 64},
        # a token for each of many conversations of different lengths: the cache's bytes
        {"name": "decode batch", "op": "decode", "seqs": 64, "longest": 8192, "queries": 1, "heads": 32, "kv": 8, "dim": 128,
         "dtype": "bf16", "page": 64},
        # one very long document
        {"name": "decode long", "op": "decode", "seqs": 1, "longest": 200001, "queries": 1, "heads": 16, "kv": 2, "dim": 128,
         "dtype": "f16", "page": 128},
        # up to five drafted tokens of each sequence at once, smaller heads, small pages
        {"name": "decode drafts", "op": "decode", "seqs": 20, "longest": 5000, "queries": 5, "heads": 28, "kv": 4, "dim": 64,
         "dtype": "bf16", "page": 16},
        # one short prompt: latency
        {"name": "prompt short", "op": "prompt", "seqs": 1, "longest": 150, "heads": 32, "kv": 8, "dim": 128, "dtype": "bf16"},
        # prompts of different lengths in one call
        {"name": "prompt packed", "op": "prompt", "seqs": 13, "longest": 2500, "heads": 28, "kv": 4, "dim": 64, "dtype": "f16"},
        # a long document: the tensor cores' rate
        {"name": "prompt long", "op": "prompt", "seqs": 1, "longest": 16384, "heads": 32, "kv": 8, "dim": 128, "dtype": "bf16"},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["qk", "store", "decode", "prompt"])
    kv = rng.choice([1, 2, 3, 4, 8])
    heads, dim = kv * rng.choice([1, 2, 4, 5, 7, 8]), rng.choice([64, 128])
    dtype, page = rng.choice(["bf16", "bf16", "f16"]), rng.choice([16, 32, 64, 128, 256])
    if op == "qk":
        append = rng.random() < 0.4
        interleaved = rng.random() < 0.3
        if not append:
            dtype = rng.choice(["f32", "f16", "bf16"])
        return {"op": op, "tokens": _spread(rng, 1, 8192 * 40 * 128 // ((heads + kv) * dim) // 2), "heads": heads, "kv": kv, "dim": dim,
                "rot": rng.choice([dim, dim, dim // 2, dim // 4]), "interleaved": interleaved, "norm": rng.random() < 0.7,
                "dtype": dtype, "append": append, **({"page": page} if append else {})}
    if op == "store":
        return {"op": op, "tokens": _spread(rng, 1, 16384 * 8 * 128 // (kv * dim)), "kv": kv, "dim": dim,
                "dtype": rng.choice(["f32", "f16", "bf16"]), "page": page}
    if op == "decode":
        longest = _spread(rng, 1, 200000)
        most = max(1, 64 * 8192 * 8 * 128 // (longest * kv * dim))
        return {"op": op, "seqs": _spread(rng, 1, min(most, 200)), "longest": longest, "queries": rng.choice([1, 1, 1, 2, 4, 7]),
                "heads": heads, "kv": kv, "dim": dim, "dtype": dtype, "page": page}
    longest = _spread(rng, 1, 12000)
    most = max(1, 8 * 16384 * 16384 // (longest * longest * heads))
    return {"op": op, "seqs": _spread(rng, 1, min(most, 40)), "longest": longest, "heads": heads, "kv": kv, "dim": dim, "dtype": dtype}


def _lengths(case):
    """The sequences' lengths, and the tokens that each asks for at its end: the longest first, the others as they fall."""
    rng = random.Random(str(sorted(case.items())))
    lens = [case["longest"]] + [_spread(rng, 1, case["longest"]) for _ in range(case["seqs"] - 1)]
    most = case.get("queries", 1)
    return lens, [min(n, most if i == 0 else rng.randint(1, most)) for i, n in enumerate(lens)]


def _starts(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _inputs(case, seed):
    """The inputs by name, on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    op, dtype = case["op"], DTYPES[case["dtype"]]
    kv, dim = case["kv"], case["dim"]
    if op == "decode":
        lens, asked = _lengths(case)
        pages = [-(-n // case["page"]) for n in lens]
        order = torch.randperm(sum(pages), generator=g, device="cuda")
        table = torch.zeros(len(lens), max(pages), dtype=torch.int32, device="cuda")
        table[torch.arange(max(pages), device="cuda")[None] < torch.tensor(pages, device="cuda")[:, None]] = order.int()
        places = sum(pages) * case["page"]
        # normed and rotated keys: some channels larger than the others; places past a sequence's end hold what an earlier one left
        loud = 1 + 1.5 * (torch.rand(kv, dim, generator=g, device="cuda") < 0.05)
        return {"q": normal(sum(asked), case["heads"], dim).to(dtype), "k": (normal(places, kv, dim) * loud).to(dtype),
                "v": normal(places, kv, dim).to(dtype), "table": table, "lengths": torch.tensor(lens, dtype=torch.int32, device="cuda"),
                "starts": torch.tensor(_starts(asked), dtype=torch.int32, device="cuda") if case["queries"] > 1 else None}
    if op == "prompt":
        lens, _ = _lengths(case)
        tokens, heads = sum(lens), case["heads"]
        # values as they lie in the product that made them, queries and keys after their norm and rotation
        both = normal(tokens, heads + 2 * kv, dim).to(dtype)
        return {"q": normal(tokens, heads, dim).to(dtype), "k": normal(tokens, kv, dim).to(dtype), "v": both[:, heads + kv:],
                "starts": torch.tensor(_starts(lens), dtype=torch.int32, device="cuda")}
    tokens = case["tokens"]
    s = {}
    if op == "store" or case["append"]:
        places = -(-2 * tokens // case["page"]) * case["page"]
        s["slots"] = torch.randperm(places, generator=g, device="cuda")[:tokens]
        s["places"] = places
    if op == "store":
        s["k"] = (3 * normal(tokens, kv, dim) + normal(kv, dim)).to(dtype)
        s["v"] = normal(tokens, kv, dim).to(dtype)
        return s
    heads, rot = case["heads"], case["rot"]
    both = (2 * normal(tokens, heads + 2 * kv, dim)).to(dtype)  # one product's output
    s["q"], s["k"], s["v"] = both[:, :heads], both[:, heads:heads + kv], both[:, heads + kv:]
    s["positions"] = torch.randint(0, 1_000_000, (1,), generator=g, device="cuda") + torch.arange(tokens, device="cuda")
    s["inv_freq"] = (10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)).float()
    s["q_weight"] = (1 + 0.2 * normal(dim)).to(dtype) if case["norm"] else None
    s["k_weight"] = (1 + 0.2 * normal(dim)).to(dtype) if case["norm"] else None
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=case)
    if "page" in case:
        page, kv, dim = case["page"], case["kv"], case["dim"]
        places = s["k"].shape[0] if case["op"] == "decode" else s["places"]
        if own:
            from paper_2007_06919_gb300 import aqd
            s["cache"] = aqd.KVCache(places // page, page, kv, dim)
            if case["op"] == "decode":
                aqd.cache_write(s["cache"], s.pop("k"), s.pop("v"), torch.arange(places, device="cuda"))
                s["workspace"] = aqd.cache_attention_workspace(s["q"], s["cache"], s["lengths"].numel())
        elif case["op"] == "decode":
            s["cache"] = [_quantised(s.pop("k").float()), _quantised(s.pop("v").float())]
        else:
            s["cache"] = [(torch.zeros(places, kv, dim // 2, dtype=torch.uint8, device="cuda"),
                           *(torch.zeros(places, kv, 1, dtype=torch.bfloat16, device="cuda") for _ in range(2))) for _ in range(2)]
    if case["op"] in ("decode", "prompt"):
        lens, asked = _lengths(case)
        s["most"] = max(asked) if case["op"] == "decode" else max(lens)
    return s


def run(state):
    op = state["case"]["op"]
    if own:
        return {"qk": _own_qk, "store": _own_store, "decode": _own_decode, "prompt": _own_prompt}[op](state)
    return {"qk": _qk, "store": _store, "decode": _decode, "prompt": _prompt}[op](state)


# ------------------------------------------------------------------ the framework's operators


def _own_qk(s):
    from paper_2007_06919_gb300 import aqd
    case = s["case"]
    more = {"v": s["v"], "cache": s["cache"], "slots": s["slots"]} if case["append"] else {}
    out = aqd.qk_norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                           interleaved=case["interleaved"], **more)
    if not case["append"]:
        return {"q": out.q, "k": out.k}
    k, v = aqd.cache_read(s["cache"], s["slots"], dtype=VALUES[case["dtype"]])
    return {"q": out.q, "k": k, "v": v}


def _own_store(s):
    from paper_2007_06919_gb300 import aqd
    aqd.cache_write(s["cache"], s["k"], s["v"], s["slots"])
    k, v = aqd.cache_read(s["cache"], s["slots"], dtype=VALUES[s["case"]["dtype"]])
    return {"k": k, "v": v}


def _own_decode(s):
    from paper_2007_06919_gb300 import aqd
    return aqd.cache_attention(s["q"], s["cache"], s["table"], s["lengths"], starts=s["starts"], workspace=s["workspace"])


def _own_prompt(s):
    from paper_2007_06919_gb300 import aqd
    return aqd.prompt_attention(s["q"], s["k"], s["v"], s["starts"])


# ------------------------------------------------------------------ the plain forms


def _up(x):
    """x, 0 or more, rounded up to a bfloat16's 8 bits."""
    return ((x.view(torch.int32) + 0xFFFF) & -0x10000).view(torch.float32)


def _quantised(x):
    """Rows of 4-bit codes, two to a byte, and each row's lowest value and step."""
    low = x.amin(-1, keepdim=True)
    low = torch.where(low < 0, -_up(-low), (low.view(torch.int32) & -0x10000).view(torch.float32))
    step = _up((x.amax(-1, keepdim=True) - low) / torch.full_like(low, 15))  # (by a number it would multiply by 1 / 15, rounded)
    codes = torch.round((x - low) / step).clamp_(0, 15).to(torch.uint8)  # ties to even
    return codes[..., ::2] + 16 * codes[..., 1::2], low.bfloat16(), step.bfloat16()


def _values(part, at):
    """The values that the cache holds at places `at`, in 32 bits."""
    packed, low, step = (t[at] for t in part)
    codes = torch.stack([packed & 15, packed >> 4], -1).flatten(-2).float()
    return codes.mul_(step.float()).add_(low.float())


def _put_and_read(s, k, v):
    dtype = VALUES[s["case"]["dtype"]]
    for part, x in zip(s["cache"], (k, v)):
        for held, new in zip(part, _quantised(x.float())):
            held[s["slots"]] = new
    k, v = (_values(part, s["slots"]).to(dtype) for part in s["cache"])
    return {"k": k, "v": v}


def _normed(x, weight):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    return x


def _rotated(x, cos, sin, rot, interleaved):
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _qk(s):
    case, dtype = s["case"], s["q"].dtype
    angle = (s["positions"].double()[:, None] * s["inv_freq"].double())[:, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    q, k = (_rotated(_normed(s[n], s[n + "_weight"]), cos, sin, case["rot"], case["interleaved"]).to(dtype) for n in "qk")
    return {"q": q, **_put_and_read(s, k, s["v"])} if case["append"] else {"q": q, "k": k}


def _store(s):
    return _put_and_read(s, s["k"], s["v"])


def _softmax(scores, seen):
    scores = scores.masked_fill_(~seen, -math.inf)
    p = scores.sub_(scores.amax(-1, keepdim=True).clamp_(min=-1e30)).exp_()
    return p.div_(p.sum(-1, keepdim=True).clamp_(min=1e-30))


def _decode(s):
    q, lens, table, page = s["q"], s["lengths"], s["table"], s["case"]["page"]
    heads, kv, dim = s["case"]["heads"], s["case"]["kv"], s["case"]["dim"]
    seqs, longest, most = lens.numel(), s["case"]["longest"], s["most"]
    t = torch.arange(longest, device=q.device)
    at = table[:, t // page].long() * page + t % page                       # [seqs, longest]
    if s["starts"] is None:
        first, n = torch.arange(seqs, device=q.device), torch.ones_like(lens)
    else:
        first, n = s["starts"][:-1].long(), s["starts"].diff()
    j = torch.arange(most, device=q.device)
    rows = (first[:, None] + j).clamp_(max=q.shape[0] - 1)                  # queries of each sequence, the last ones empty
    g = heads // kv
    x = q[rows].float().view(seqs, most, kv, g, dim).permute(0, 2, 1, 3, 4).reshape(seqs, kv, most * g, dim)
    scores = x @ _values(s["cache"][0], at).permute(0, 2, 3, 1) * (1 / math.sqrt(dim))
    seen = t[None, None] < (lens[:, None] - n[:, None] + j + 1)[..., None]  # [seqs, most, longest]
    p = _softmax(scores.view(seqs, kv, most, g, longest), seen[:, None, :, None])
    o = p.view(seqs, kv, most * g, longest) @ _values(s["cache"][1], at).permute(0, 2, 1, 3)
    o = o.view(seqs, kv, most, g, dim).permute(0, 2, 1, 3, 4).reshape(seqs * most, heads, dim)
    if s["starts"] is None:
        return o.to(q.dtype)
    out = torch.empty_like(q)
    kept = (j < n[:, None])
    out[rows[kept]] = o[kept.flatten()].to(q.dtype)
    return out


def _prompt(s):
    q, k, v, starts = s["q"], s["k"], s["v"], s["starts"].long()
    heads, kv, dim = s["case"]["heads"], s["case"]["kv"], s["case"]["dim"]
    seqs, most = starts.numel() - 1, s["most"]
    t = torch.arange(most, device=q.device)
    rows = (starts[:-1, None] + t).clamp_(max=q.shape[0] - 1)               # [seqs, most], padded
    x, y, z = (a[rows].float().transpose(1, 2) for a in (q, k, v))          # [seqs, heads, most, dim]
    scores = x.reshape(seqs, kv, -1, dim) @ y.transpose(2, 3) * (1 / math.sqrt(dim))
    p = _softmax(scores.view(seqs, heads, most, most), t[:, None] >= t)
    o = (p.view(seqs, kv, -1, most) @ z).view(seqs, heads, most, dim).transpose(1, 2).to(q.dtype)
    kept = t < starts.diff()[:, None]
    out = torch.empty_like(q)
    out[rows[kept]] = o[kept]
    return out


# ------------------------------------------------------------------ work and exact values


def work(case):
    op, dim, kv, e = case["op"], case["dim"], case["kv"], SIZE[case["dtype"]]
    row = dim // 2 + 4  # codes, lowest value and step
    if op == "qk":
        x = case["tokens"] * (case["heads"] + kv) * dim
        more = case["tokens"] * kv * dim
        if case["append"]:  # keys and values into the cache, and from there
            return {"bytes": x * e + case["tokens"] * case["heads"] * dim * e + more * e + case["tokens"] * kv * 4 * row + 4 * more,
                    "flops": 10 * x + 16 * more}
        return {"bytes": 2 * x * e + 8 * case["tokens"], "flops": 10 * x}
    if op == "store":
        x = 2 * case["tokens"] * kv
        return {"bytes": x * (dim * e + 2 * row + dim * 2) + 16 * case["tokens"], "flops": 8 * x * dim}
    lens, asked = _lengths(case)
    if op == "decode":
        pairs = sum(n * (m - n) + n * (n + 1) // 2 for m, n in zip(lens, asked))
        return {"bytes": sum(lens) * kv * 2 * row + 2 * sum(asked) * case["heads"] * dim * e,
                "flops": 4 * pairs * case["heads"] * dim}
    pairs = sum(n * (n + 1) // 2 for n in lens)
    return {"bytes": sum(lens) * 2 * (case["heads"] + kv) * dim * e, "flops": 4 * pairs * case["heads"] * dim}


def _held(x):
    """What the cache holds for rows x, from the definition in 64 bits."""
    x = x.double()
    lowest, highest = x.aminmax(dim=-1, keepdim=True)
    low = lowest.bfloat16()
    low = torch.where(low.double() > lowest, torch.nextafter(low, torch.full_like(low, -math.inf)), low).double()
    each = (highest - low) / torch.full_like(low, 15)
    step = each.bfloat16()
    step = torch.where(step.double() < each, torch.nextafter(step, torch.full_like(step, math.inf)), step).double()
    t = (x - low) / step
    code = torch.floor(t + 0.5)
    code -= ((code - t == 0.5) & (code % 2 == 1)).double()  # halfway: the even one
    return low + step * code.clamp(0, 15)


def _attended(q, k, v, before):
    """q [n, heads, dim] over k and v [m, kv, dim] in 64 bits; query i sees the first before + i + 1 of them."""
    n, heads, dim = q.shape
    out = torch.empty(n, heads, dim, dtype=torch.float64, device=q.device)
    block = 2048
    for h in range(heads):
        keys, vals = (a[:, h * a.shape[1] // heads].double() for a in (k, v))
        for a in range(0, n, block):
            b = min(n, a + block)
            see = before + b
            scores = torch.mm(q[a:b, h].double(), keys[:see].t()) / dim ** 0.5
            places = torch.arange(see, device=q.device)
            scores[places > before + torch.arange(a, b, device=q.device)[:, None]] = -math.inf
            out[a:b, h] = torch.mm(torch.softmax(scores, dim=1), vals[:see])
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    op, dtype = case["op"], DTYPES[case["dtype"]]
    if op == "store":
        return {"k": _held(s["k"]), "v": _held(s["v"])}
    if op == "qk":
        out = {}
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                           torch.outer(s["positions"].double(), s["inv_freq"].double()))[:, None]
        for name in "qk":
            x = s[name].double()
            if case["norm"]:
                x = x / (x.pow(2).mean(dim=-1, keepdim=True) + EPS).sqrt() * s[name + "_weight"].double()
            x = x.clone()
            r = case["rot"]
            first, second = (slice(0, r, 2), slice(1, r, 2)) if case["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
            y = torch.complex(x[..., first], x[..., second]) * turn
            x[..., first], x[..., second] = y.real, y.imag
            out[name] = x
        return {"q": out["q"], "k": _held(out["k"].to(dtype)), "v": _held(s["v"])} if case["append"] else out
    if op == "prompt":
        at = s["starts"].tolist()
        return torch.cat([_attended(s["q"][a:b], s["k"][a:b], s["v"][a:b], 0) for a, b in zip(at, at[1:])])
    lens, asked = _lengths(case)
    at, out = _starts(asked), []
    for i, n in enumerate(lens):
        t = torch.arange(n, device="cuda")
        places = s["table"][i].long()[t // case["page"]] * case["page"] + t % case["page"]
        out.append(_attended(s["q"][at[i]:at[i + 1]], _held(s["k"][places]), _held(s["v"][places]), n - asked[i]))
    return torch.cat(out)
