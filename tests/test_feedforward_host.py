"""What the decoder's blocks and head hand to the operators, on the CPU: fakes stand for the operators and record."""
from types import SimpleNamespace

import pytest
import torch

from paper_2007_06919_gb300 import aqd, feedforward


class Stream:
    """A CUDA stream as the binding sees it."""
    def __init__(self, handle):
        self.cuda_stream, self.device, self.waited = handle, torch.device("cuda", 0), 0

    def synchronize(self):
        self.waited += 1


class Kept:
    """Memory of the model's own, and the streams that the allocator was told of."""
    def __init__(self, *shape):
        self.shape, self.streams = torch.Size(shape), []

    def record_stream(self, s):
        self.streams.append(s)


@pytest.fixture
def record(monkeypatch):
    """The products' (tokens, weights, workspace, stream) in turn; every workspace knows its size and stream, and stays alive."""
    calls, default = [], Stream(0)

    def codes(shape):
        return aqd.RowCodes(torch.zeros(shape, dtype=torch.int8), torch.zeros(shape[:-1]), None, torch.zeros(shape))

    def linear(x, xs, w, *, out_dtype, workspace=None, stream=None):
        calls.append((x.numel() // w.k, w, workspace, stream))
        return torch.zeros(*x.shape[:-1], w.n)

    monkeypatch.setattr(feedforward, "aqd", SimpleNamespace(
        LinearWeights=SimpleNamespace(from_float=lambda w, stream=None: SimpleNamespace(
            n=w.shape[0], k=w.shape[1], device=w.device, index=0, scales=Kept(w.shape[0]), prepared=Kept(1))),
        linear_workspace=lambda m, *w, stream=None: SimpleNamespace(m=m, k=max(v.k for v in w), stream=stream),
        rms_norm_quant=lambda x, w, *, eps, residual=None, stream=None: codes(x.shape),
        gated_act_quant=lambda g, u, *, act, stream=None: codes(g.shape),
        linear_int8=linear, _stream=lambda s=None: (s or default).cuda_stream))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: default)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return SimpleNamespace(calls=calls, default=default)


def decoder(tokens, d=32, hidden=48, vocab=70):
    def part(h, v):
        return torch.zeros(h, v)
    blocks = [feedforward.FeedForward(Kept(d), part(hidden, d), part(hidden, d), part(d, hidden), tokens=tokens) for _ in range(2)]
    return feedforward.Decoder(blocks, feedforward.Head(Kept(d), part(vocab, d), tokens=tokens))


def test_no_workspace_is_shared_by_calls_on_several_streams(record):
    net, streams = decoder(40), [Stream(1), Stream(2), None]
    for s in streams:
        net(torch.zeros(40, 32), stream=s)
    assert len(record.calls) == 15
    spaces = [ws for _, _, ws, _ in record.calls]
    assert all(ws is not None for ws in spaces)
    assert all(a is not b for i, a in enumerate(spaces) for j, b in enumerate(spaces) if i // 5 != j // 5)
    assert all(ws.stream is s for _, _, ws, s in record.calls)


@pytest.mark.parametrize("tokens", [1, 16, 17, 300, 5000])
def test_a_workspace_is_as_large_as_its_calls_tokens_need(record, tokens):
    """Whatever the model was built for; a product of more than 16 tokens without one runs on the kernels for few."""
    net = decoder(4)
    for shape in ((tokens, 32), (1, tokens, 32)):
        net(torch.zeros(shape))
    for m, w, ws, _ in record.calls:
        assert m == tokens
        assert (ws is None and m <= 16) or (ws.m >= m and ws.k >= w.k)


@pytest.mark.parametrize("tokens", [3, 40])
def test_blocks_and_heads_alone(record, tokens):
    net = decoder(1, d=30)
    for s in (Stream(1), Stream(2)):
        net.blocks[0](torch.zeros(tokens, 30), stream=s)
        net.head(torch.zeros(tokens, 30), stream=s)
    assert len(record.calls) == 6 and all(ws.m >= m and ws.k >= w.k and ws.stream is s for m, w, ws, s in record.calls)


def test_the_weights_are_there_for_every_stream(record):
    """Prepared on the stream current then, they are complete before a call may come on another."""
    net = decoder(4)
    assert record.default.waited >= len(net.blocks) + 1


def test_memory_in_use_on_another_stream_is_not_given_away(record):
    """A model that is dropped while another stream still reads its weights."""
    net, s = decoder(4), Stream(5)
    kept = [t for part in net.blocks + [net.head] for t in (part.norm, *(v for w in vars(part).values() if hasattr(w, "prepared")
                                                                           for v in (w.prepared, w.scales)))]
    assert len(kept) == 2 * 5 + 3
    net(torch.zeros(4, 32))
    assert not any(t.streams for t in kept)
    for _ in range(3):
        net(torch.zeros(4, 32), stream=s)
    assert all(t.streams == [s] for t in kept)


def test_few_tokens_of_odd_rows_have_a_workspace(record):
    decoder(4, d=30, hidden=47)(torch.zeros(3, 30))
    assert all(ws is not None and ws.m >= 3 for _, _, ws, _ in record.calls)
