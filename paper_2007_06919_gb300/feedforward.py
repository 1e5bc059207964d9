"""The 8-bit part of a decoder on the GPU: feed-forward blocks and an output head whose products are integer, and the
distillation of the head from a float teacher of which each token's top logits are kept.

A block is three row passes and products on one stream: norm of x + residual to 8-bit codes (the sum goes on as the next residual),
the gate and up products as one product with their rows stacked, the gated activation to codes, the down product.
Products are exact integer sums with a scale per token and per output channel; no value between two launches is
wider than 16 bits but the scales. A head is a norm and one product.

What training reaches here is the head's scale per vocabulary entry: with logits y = s_v a, dL/d(ln s_v) = sum over tokens of
(dL/dy) y, so a step multiplies the scale (it stays positive), and the prepared codes stay as they are.

``python -m paper_2007_06919_gb300.feedforward`` distils a small student of a random float model and prints its loss.
"""
from __future__ import annotations

import torch

from . import aqd


def _workspace(m: int, layers, stream):
    """A workspace for one call of a model: of that call's stream alone, since calls on several streams may overlap, and as large as its own
    tokens need. The layers' products follow one another, so they share it. None for codes that products read where they lie (up to 16 rows, each
    on 16 bytes)."""
    if m > 16 or (m > 1 and any(w.k % 16 for w in layers)):
        return aqd.linear_workspace(m, *layers, stream=stream)
    return None


class _Part:
    """Weights that calls on any stream read, in the memory of the stream current at construction."""

    def _keep(self, norm: torch.Tensor, *layers):
        self._memory = [norm] + [t for w in layers for t in (w.prepared, w.scales)]
        self._readers = {aqd._stream()}
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream().synchronize()  # prepared before the first call, wherever that comes

    def _read_on(self, stream):
        """Keeps the weights' memory, once they are dropped, until this stream has finished with it."""
        handle = aqd._stream(stream)
        if handle not in self._readers:
            for t in self._memory:
                t.record_stream(torch.cuda.current_stream() if stream is None else stream)
            self._readers.add(handle)


class FeedForward(_Part):
    """One block: norm weight [d], gate and up [hidden, d], down [d, hidden] in floating point; the products' weights
    are quantized here. Calls may bring any number of tokens, on several streams at a time. (tokens has no effect: a workspace is
    taken for each call.)"""

    def __init__(self, norm: torch.Tensor, gate: torch.Tensor, up: torch.Tensor, down: torch.Tensor, *, act: str = "silu",
                 eps: float = 1e-6, tokens: int = 1):
        if gate.shape != up.shape or down.shape != gate.shape[::-1] or norm.shape != gate.shape[1:]:
            raise ValueError("gate and up must be [hidden, d], down [d, hidden], norm [d]")
        self.norm, self.act, self.eps, self.tokens, self.hidden = norm, act, eps, tokens, gate.shape[0]
        self.both = aqd.LinearWeights.from_float(torch.cat([gate, up]))
        self.down = aqd.LinearWeights.from_float(down)
        self._keep(norm, self.both, self.down)

    def __call__(self, x: torch.Tensor, residual: torch.Tensor | None = None, stream=None, workspace=None):
        """(block's output, x + residual) of tokens x [..., d]: the two are the next norm's x and residual. workspace: one for
        these tokens and both layers (linear_workspace) that no call on another stream uses meanwhile; the call takes one where none is given."""
        self._read_on(stream)
        if workspace is None:
            workspace = _workspace(x.numel() // self.both.k, (self.both, self.down), stream)
        q = aqd.rms_norm_quant(x, self.norm, eps=self.eps, residual=residual, stream=stream)
        both = aqd.linear_int8(q.codes, q.scales, self.both, out_dtype=x.dtype, workspace=workspace, stream=stream)
        h = aqd.gated_act_quant(both[..., :self.hidden], both[..., self.hidden:], act=self.act, stream=stream)
        y = aqd.linear_int8(h.codes, h.scales, self.down, out_dtype=x.dtype, workspace=workspace, stream=stream)
        return y, x if residual is None else q.summed


class Head(_Part):
    """Norm weight [d] and a projection [vocab, d] to logits; calls and tokens as a block's."""

    def __init__(self, norm: torch.Tensor, weight: torch.Tensor, *, eps: float = 1e-6, tokens: int = 1):
        self.norm, self.eps = norm, eps
        self.proj = aqd.LinearWeights.from_float(weight)
        self._keep(norm, self.proj)

    def __call__(self, x: torch.Tensor, residual: torch.Tensor | None = None, stream=None, workspace=None) -> torch.Tensor:
        self._read_on(stream)
        if workspace is None:
            workspace = _workspace(x.numel() // self.proj.k, (self.proj,), stream)
        q = aqd.rms_norm_quant(x, self.norm, eps=self.eps, residual=residual, stream=stream)
        return aqd.linear_int8(q.codes, q.scales, self.proj, out_dtype=x.dtype, workspace=workspace, stream=stream)

    def distill(self, logits: torch.Tensor, index: torch.Tensor, teacher: torch.Tensor, *, tau: float = 1.0,
                row_weight: torch.Tensor | None = None, rate: float = 0.0):
        """The tokens' losses against a teacher's top logits and the losses' gradient by the logarithms of the scales [vocab];
        rate > 0: a gradient step on these. On the current stream."""
        out = aqd.distill_topk(logits, index, teacher, tau=tau, row_weight=row_weight, grad=True)
        vocab = logits.shape[-1]
        grad = out.grad.view(-1, vocab)
        # a gradient of 0 adds nothing, whatever the logit: of a token of weight 0 it may be a NaN, of a place that a mask rules out -infinity
        slope = (grad.float() * logits.reshape(-1, vocab).float()).masked_fill_(grad == 0, 0.0).sum(0)
        if rate:
            self.proj.scales.mul_(torch.exp(-rate * slope))
        return out.loss, slope


class Decoder:
    """Feed-forward blocks and a head in sequence."""

    def __init__(self, blocks: list[FeedForward], head: Head):
        self.blocks, self.head = blocks, head

    def __call__(self, x: torch.Tensor, stream=None) -> torch.Tensor:
        """Logits [..., vocab] of tokens x [..., d]."""
        layers = [w for block in self.blocks for w in (block.both, block.down)] + [self.head.proj]
        ws = _workspace(x.numel() // layers[0].k, layers, stream)
        residual = None
        for block in self.blocks:
            x, residual = block(x, residual, stream=stream, workspace=ws)
        return self.head(x, residual, stream=stream, workspace=ws)


def main():
    torch.manual_seed(0)
    d, hidden, vocab, tokens, top = 512, 1024, 8192, 256, 32

    def weight(n, k):
        return torch.randn(n, k, device="cuda") / k ** 0.5

    ones = torch.ones(d, device="cuda", dtype=torch.bfloat16)
    w = [(weight(hidden, d), weight(hidden, d), weight(d, hidden)) for _ in range(2)]
    out = 4 * weight(vocab, d)
    student = Decoder([FeedForward(ones, *b, tokens=tokens) for b in w], Head(ones, out, tokens=tokens))
    x = torch.randn(tokens, d, device="cuda", dtype=torch.bfloat16)
    # the teacher: the same model in floating point, its vocabulary's scales moved
    y, r = x.float(), torch.zeros(tokens, d, device="cuda")

    def rms(t):
        return t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6)

    for gate, up, down in w:
        r = r + y
        h = rms(r)
        y = (torch.nn.functional.silu(h @ gate.T) * (h @ up.T)) @ down.T
    teacher = (rms(r + y) @ out.T * (1 + 0.2 * torch.randn(vocab, device="cuda"))).topk(top)
    for step in range(31):
        loss, _ = student.head.distill(student(x), teacher.indices, teacher.values, rate=0.004)
        if step % 10 == 0:
            print(f"step {step:2d}: loss per token {loss.mean().item():.4f}")


if __name__ == "__main__":
    main()
