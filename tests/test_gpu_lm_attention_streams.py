"""The decoder's attention blocks on other streams than the current one."""
import pytest
import torch

from paper_2007_06919_gb300 import aqd
from paper_2007_06919_gb300.attention import Sequences
from test_gpu_lm_attention_decoder import model
from test_gpu_lm_streams import together

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def started(net, x, lens, stream=None, keep=None):
    """Sequences of these lengths, their caches, and the prompts' logits."""
    seqs, caches = Sequences(20, 16, 8), net.caches(20, 16)
    for c in caches:
        c.data.zero_()
    for s in range(len(lens)):
        seqs.add(s)
    torch.cuda.synchronize()
    return seqs, caches, net(x, seqs.extend(list(range(len(lens))), lens), caches, stream=stream)


def test_calls_that_overlap():
    """Prompts and steps of four sets of sequences, a stream each, at once."""
    net, _, _, _ = model(7, 256, 512, 1000, 4, 2, 64, 2)
    torch.manual_seed(1)
    xs = [(torch.randn(60, 256, device="cuda", dtype=BF16), torch.randn(2, 256, device="cuda", dtype=BF16)) for _ in range(4)]

    def both(p, x, s=None):
        seqs, caches, first = started(net, p, [45, 15], s)
        return first, net(x, seqs.extend([0, 1], [1, 1]), caches, stream=s), caches

    want = [both(*x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(3):
        made = []
        for _ in xs:
            seqs, caches = Sequences(20, 16, 8), net.caches(20, 16)
            for c in caches:
                c.data.zero_()
            seqs.add(0), seqs.add(1)
            made.append((caches, seqs.extend([0, 1], [45, 15]), seqs.extend([0, 1], [1, 1])))
        torch.cuda.synchronize()
        got = together(streams, [lambda s, x=x, m=m: (net(x[0], m[1], m[0], stream=s), net(x[1], m[2], m[0], stream=s)) for x, m in zip(xs, made)])
        for g, w, m in zip(got, want, made):
            assert torch.equal(g[0], w[0]) and torch.equal(g[1], w[1]) and all(torch.equal(a.data, b.data) for a, b in zip(m[0], w[2]))
    assert aqd.device_status() == 0


@pytest.mark.parametrize("current", [False, True])
def test_tokens_dropped_while_a_stream_still_reads_them(current):
    """Positions, slots, lengths and table of a call on another stream, dropped when it returns: later tensors do not take their memory before it has run. `current`: the
    stream is the current one at the call, and not when the tokens were made."""
    net, _, _, _ = model(8, 256, 512, 1000, 4, 2, 64, 2)
    x, steps = torch.randn(60, 256, device="cuda", dtype=BF16), torch.randn(3, 2, 256, device="cuda", dtype=BF16)
    seqs, caches, first = started(net, x, [45, 15])
    want = [first] + [net(t, seqs.extend([0, 1], [1, 1]), caches) for t in steps]
    held = [c.data.clone() for c in caches]

    seqs, caches = Sequences(20, 16, 8), net.caches(20, 16)
    for c in caches:
        c.data.zero_()
    seqs.add(0), seqs.add(1)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(200_000_000)
    got, taken = [], []
    for t, counts in [(x, [45, 15])] + [(t, [1, 1]) for t in steps]:
        tokens = seqs.extend([0, 1], counts)
        sizes = {a.numel() * a.element_size() for a in (tokens.starts, tokens.positions, tokens.slots, tokens.lengths, tokens.table)}
        if current:
            with torch.cuda.stream(s):
                got.append(net(t, tokens, caches))
        else:
            got.append(net(t, tokens, caches, stream=s))
        del tokens
        taken += [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(8)]
    assert not s.query()  # the stream had not begun
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want)) and all(torch.equal(c.data, h) for c, h in zip(caches, held)) and len(taken) > 0
