"""Cases of the 8-bit language-model operators and of the distillation loss: inputs, plain forms, exact values.

Operators (``op``):
  norm     residual addition, root-mean-square norm, 8-bit codes with one scale per token
  gated    gated activation between two products, 8-bit codes with one scale per token
  linear   product of 8-bit codes with a scale per token and per output channel
  distill  distillation from a teacher's top logits: the loss, a training step (loss and gradient), or the
           gradient from a saved normalizer
Codes are returned as the values they stand for (code x scale), in 16 bits: the inputs' type, or bfloat16 where a
model keeps these in 32 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
VALUES = {"f32": torch.bfloat16, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


def listed():
    return [
        # one decoded token through a block's norm: latency
        {"name": "norm one token", "op": "norm", "tokens": 1, "width": 4096, "dtype": "bf16", "residual": True},
        # a prompt's tokens through the same norm: bandwidth
        {"name": "norm prompt", "op": "norm", "tokens": 4096, "width": 4096, "dtype": "bf16", "residual": True},
        # the first norm of a small model kept in 32 bits: nothing to add, an odd width
        {"name": "norm odd f32", "op": "norm", "tokens": 777, "width": 1537, "dtype": "f32", "residual": False},
        # a batch of decoded tokens between a feed-forward's products
        {"name": "gated decode", "op": "gated", "tokens": 16, "width": 12288, "dtype": "bf16", "act": "silu"},
        # a prompt between them, the other activation
        {"name": "gated prompt", "op": "gated", "tokens": 4096, "width": 12288, "dtype": "f16", "act": "gelu_tanh"},
        # one decoded token: the weights' bytes
        {"name": "linear one token", "op": "linear", "tokens": 1, "n": 4096, "k": 4096, "dtype": "bf16", "bias": False},
        # a batch of decoded tokens on a wide layer: the weights' bytes, more sums for each
        {"name": "linear batch", "op": "linear", "tokens": 24, "n": 12288, "k": 4096, "dtype": "bf16", "bias": False},
        # a short prompt on a layer of uneven sizes, with a bias
        {"name": "linear ragged", "op": "linear", "tokens": 333, "n": 1000, "k": 2050, "dtype": "f32", "bias": True},
        # a long prompt: the tensor cores' rate
        {"name": "linear prompt", "op": "linear", "tokens": 8192, "n": 12288, "k": 4096, "dtype": "bf16", "bias": False},
        # how far a quantized model is from its teacher: the loss alone, 32-bit logits
        {"name": "distill loss", "op": "distill", "mode": "loss", "tokens": 512, "vocab": 32000, "top": 16, "dtype": "f32", "tau": 1.0},
        # a training step on a large vocabulary: loss and gradient
        {"name": "distill step", "op": "distill", "mode": "step", "tokens": 2048, "vocab": 131072, "top": 64, "dtype": "bf16", "tau": 2.0},
        # the gradient of a small batch on an odd vocabulary, from the saved normalizer
        {"name": "distill backward", "op": "distill", "mode": "backward", "tokens": 100, "vocab": 50001, "top": 20, "dtype": "f16", "tau": 1.5},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def _size(rng, lo, hi):
    """The same; about half of them multiples of 64, the others as they fall, odd ones among them."""
    v = _spread(rng, lo, hi)
    return v if rng.random() < 0.5 else max(lo, v // 64 * 64)


def draw(rng):
    op = rng.choice(["norm", "gated", "linear", "distill"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    if op == "norm":
        width = _size(rng, 64, 16384)
        return {"op": op, "tokens": _spread(rng, 1, min(8192, 4096 * 4096 // width)), "width": width, "dtype": dtype,
                "residual": rng.random() < 0.7}
    if op == "gated":
        width = _size(rng, 64, 32768)
        return {"op": op, "tokens": _spread(rng, 1, min(8192, 4096 * 12288 // width)), "width": width, "dtype": dtype,
                "act": rng.choice(["silu", "gelu_tanh"])}
    if op == "linear":
        n, k = _size(rng, 16, 16384), _size(rng, 16, 16384)
        return {"op": op, "tokens": _spread(rng, 1, min(8192, 8192 * 12288 * 4096 // (n * k))), "n": n, "k": k,
                "dtype": dtype, "bias": rng.random() < 0.4}
    vocab = _size(rng, 500, 200000)
    return {"op": op, "mode": rng.choice(["loss", "step", "backward"]), "vocab": vocab,
            "tokens": _spread(rng, 1, min(4096, 1024 * 131072 // vocab)), "top": _spread(rng, 1, 128), "dtype": dtype,
            "tau": rng.choice([1.0, 1.5, 2.0, 4.0])}


def _inputs(case, seed):
    """The inputs by name, on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    op, m = case["op"], case["tokens"]
    if op == "linear":
        n, k = case["n"], case["k"]
        s = {"w": (normal(n, k) * 32).round_().clamp_(-127, 127).to(torch.int8),
             "x": (normal(m, k) * 32).round_().clamp_(-127, 127).to(torch.int8)}
        s["x_scale"] = 0.01 + 0.05 * uniform(m)
        s["w_scale"] = (0.5 + uniform(n)) / (32 * math.sqrt(k))
        s["bias"] = normal(n) if case["bias"] else None
        return s
    dtype = DTYPES[case["dtype"]]
    if op == "norm":
        d = case["width"]
        # activations with a few channels much larger than the others
        spread = torch.where(uniform(d) < 0.01, 20.0, 1.0)
        return {"x": (normal(m, d) * spread).to(dtype), "weight": (1 + 0.2 * normal(d)).to(dtype),
                "residual": (2 * normal(m, d)).to(dtype) if case["residual"] else None}
    if op == "gated":
        # one product's output: the gates in the first half of a row, the others in the second
        return {"both": (1.5 * normal(m, 2 * case["width"])).to(dtype)}
    logits = (3 * normal(m, case["vocab"])).to(dtype)
    # a teacher that agrees with the student but for noise
    top = (logits.float() + normal(m, case["vocab"])).topk(case["top"], dim=1)
    s = {"logits": logits, "index": top.indices, "teacher": top.values.contiguous(),
         "weight": torch.where(uniform(m) < 0.1, 0.0, 1.0) / m}  # a tenth of the tokens is padding
    if case["mode"] == "backward":
        s["lse"] = (logits.double() / case["tau"]).logsumexp(1).float()
    return s


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case)
    if own and case["op"] == "linear":
        from paper_2007_06919_gb300 import aqd
        # the layer's weights as a program keeps them, and its workspace
        state["layer"] = aqd.LinearWeights(state.pop("w"), state["w_scale"])
        state["workspace"] = aqd.linear_workspace(case["tokens"], state["layer"])
    return state


def run(state):
    op = state["case"]["op"]
    if own:
        return {"norm": _own_norm, "gated": _own_gated, "linear": _own_linear, "distill": _own_distill}[op](state)
    return {"norm": _norm, "gated": _gated, "linear": _linear, "distill": _distill}[op](state)


# ------------------------------------------------------------------ the framework's operators


def _own_norm(s):
    from paper_2007_06919_gb300 import aqd
    q = aqd.rms_norm_quant(s["x"], s["weight"], eps=EPS, residual=s["residual"], values=VALUES[s["case"]["dtype"]])
    return {"values": q.values, "scales": q.scales, "sum": q.summed}


def _own_gated(s):
    from paper_2007_06919_gb300 import aqd
    gate, up = s["both"].chunk(2, dim=1)
    q = aqd.gated_act_quant(gate, up, act=s["case"]["act"], values=VALUES[s["case"]["dtype"]])
    return {"values": q.values, "scales": q.scales}


def _own_linear(s):
    from paper_2007_06919_gb300 import aqd
    return aqd.linear_int8(s["x"], s["x_scale"], s["layer"], bias=s["bias"], out_dtype=DTYPES[s["case"]["dtype"]],
                           workspace=s["workspace"])


def _own_distill(s):
    from paper_2007_06919_gb300 import aqd
    tau, mode = s["case"]["tau"], s["case"]["mode"]
    if mode == "backward":
        return aqd.distill_topk_backward(s["logits"], s["index"], s["teacher"], s["lse"], s["weight"], tau=tau)
    out = aqd.distill_topk(s["logits"], s["index"], s["teacher"], tau=tau, row_weight=s["weight"], grad=mode == "step")
    return {"loss": out.loss, "lse": out.lse, "grad": out.grad}


# ------------------------------------------------------------------ the plain forms


def _codes(u, dtype):
    """(the values that 8-bit codes of the rows of u stand for, their scales)."""
    top = u.abs().amax(1, keepdim=True)
    codes = torch.round(u * (127.0 / top))
    scales = top / 127.0
    return (codes * scales).to(dtype), scales.squeeze(1)


def _norm(s):
    dtype = s["x"].dtype
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    u = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["weight"].float()
    values, scales = _codes(u, VALUES[s["case"]["dtype"]])
    return {"values": values, "scales": scales, "sum": h.to(dtype) if s["residual"] is not None else None}


def _gated(s):
    gate, up = (v.float() for v in s["both"].chunk(2, dim=1))
    if s["case"]["act"] == "silu":
        act = gate / (1 + torch.exp(-gate))
    else:
        act = 0.5 * gate * (1 + torch.tanh(math.sqrt(2 / math.pi) * (gate + 0.044715 * gate * gate * gate)))
    values, scales = _codes(act * up, VALUES[s["case"]["dtype"]])
    return {"values": values, "scales": scales}


def _linear(s):
    y = (s["x"].float() @ s["w"].float().T) * s["x_scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(DTYPES[s["case"]["dtype"]])


def _distill(s):
    tau, mode = s["case"]["tau"], s["case"]["mode"]
    z = s["logits"].float() / tau
    t = s["teacher"].float() / tau
    e = torch.exp(t - t.amax(1, keepdim=True))
    p = e / e.sum(1, keepdim=True)
    if mode == "backward":
        lse = s["lse"]
    else:
        top = z.amax(1)
        lse = top + torch.log(torch.exp(z - top[:, None]).sum(1))
        loss = s["weight"] * (p * (torch.log(p) - z.gather(1, s["index"]) + lse[:, None])).sum(1)
        if mode == "loss":
            return {"loss": loss, "lse": lse, "grad": None}
    q = torch.exp(z - lse[:, None])
    grad = q.scatter_add_(1, s["index"], -p) * (s["weight"] / tau)[:, None]
    grad = grad.to(s["logits"].dtype)
    return grad if mode == "backward" else {"loss": loss, "lse": lse, "grad": grad}


# ------------------------------------------------------------------ work and exact values


def work(case):
    op, m = case["op"], case["tokens"]
    e = SIZE[case["dtype"]]
    if op == "norm":
        d = case["width"]
        # inputs, the sum, codes and their values; the weights; the scales
        each = e * (3 if case["residual"] else 1) + 1 + 2
        return {"bytes": m * d * each + d * e + 4 * m, "flops": 8 * m * d}
    if op == "gated":
        return {"bytes": m * case["width"] * (2 * e + 1 + 2) + 4 * m, "flops": 12 * m * case["width"]}
    if op == "linear":
        n, k = case["n"], case["k"]
        return {"bytes": m * k + n * k + e * m * n + 4 * (m + n) + (4 * n if case["bias"] else 0), "flops": 2 * m * n * k}
    v = case["vocab"]
    return {"bytes": m * v * e * (1 if case["mode"] == "loss" else 2) + 12 * m * case["top"] + 12 * m, "flops": 8 * m * v}


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]

    def rounded(u):
        largest = u.abs().max(dim=1, keepdim=True).values
        step = largest / 127
        return torch.floor(u / step + 0.5) * step, step[:, 0]

    if op == "norm":
        total = s["x"].double()
        if s["residual"] is not None:
            total = total + s["residual"].double()
        size = ((total ** 2).sum(dim=1, keepdim=True) / total.shape[1] + EPS) ** 0.5
        values, scales = rounded(total / size * s["weight"].double())
        return {"values": values, "scales": scales, "sum": None if s["residual"] is None else total}
    if op == "gated":
        d = case["width"]
        gate, up = s["both"][:, :d].double(), s["both"][:, d:].double()
        if case["act"] == "silu":
            u = gate * torch.sigmoid(gate) * up
        else:
            # (1 + tanh z) / 2 is the logistic function at 2 z
            u = gate * torch.sigmoid((gate + 0.044715 * gate ** 3) * math.sqrt(8 / math.pi)) * up
        values, scales = rounded(u)
        return {"values": values, "scales": scales}
    if op == "linear":
        # sums of products below 2^14 over at most 2^14 terms: whole in 64 bits
        y = torch.mm(s["x"].double(), s["w"].double().t())
        y = torch.einsum("mn,m,n->mn", y, s["x_scale"].double(), s["w_scale"].double())
        return y if s["bias"] is None else y + s["bias"].double()
    tau, mode = case["tau"], case["mode"]
    logq = torch.log_softmax(s["logits"].double() / tau, dim=1)
    logp = torch.log_softmax(s["teacher"].double() / tau, dim=1)
    weight = s["weight"].double()
    if mode == "backward":
        logq = s["logits"].double() / tau - s["lse"].double()[:, None]
    grad = None
    if mode != "loss":
        grad = logq.exp()
        rows = torch.arange(case["tokens"], device="cuda")[:, None].expand_as(s["index"])
        grad.index_put_((rows, s["index"]), -logp.exp(), accumulate=True)
        grad *= weight[:, None] / tau
        if mode == "backward":
            return grad
    loss = weight * torch.nn.functional.kl_div(logq.gather(1, s["index"]), logp, reduction="none", log_target=True).sum(dim=1)
    lse = torch.logsumexp(s["logits"].double() / tau, dim=1)
    return {"loss": loss, "lse": lse, "grad": grad}
