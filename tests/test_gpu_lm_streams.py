"""One decoder on several streams at a time, and with more tokens than it was told of."""
import pytest
import torch

from paper_2007_06919_gb300 import aqd
from test_gpu_lm_decoder import model

pytestmark = pytest.mark.gpu


def together(streams, calls):
    """Every call on its stream, all held back until the last one is in its queue."""
    gate = torch.cuda.Event()
    torch.cuda._sleep(20_000_000)  # about 10 ms
    gate.record()
    out = []
    for s, call in zip(streams, calls):
        s.wait_event(gate)
        out.append(call(s))
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("d", [256, 250])
@pytest.mark.parametrize("tokens", [7, 40, 300, 1500])
def test_calls_that_overlap(tokens, d):
    net, _, _, x = model(11, d, 512, 1000, 2, tokens)
    xs = [x, x.flip(0).contiguous(), -x, 2 * x.roll(1, 1)]
    want = [net(v) for v in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(5):
        got = together(streams, [lambda s, v=v: net(v, stream=s) for v in xs])
        for g, w in zip(got, want):
            assert torch.equal(g, w)
    assert aqd.device_status() == 0


@pytest.mark.parametrize("tokens", [40, 700])
def test_more_tokens_than_stated(tokens):
    net, _, _, x = model(12, 256, 512, 1000, 1, tokens)
    small, _, _, _ = model(12, 256, 512, 1000, 1, 1)
    assert torch.equal(net(x), small(x))
    torch.cuda.synchronize()


def test_first_call_on_another_stream():
    want = model(13, 512, 1024, 2000, 2, 40)[0]
    x = torch.randn(40, 512, device="cuda").bfloat16()
    want = want(x)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)  # the weights are prepared behind this
    net = model(13, 512, 1024, 2000, 2, 40)[0]
    got = net(x, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    torch.cuda.synchronize()


def test_a_model_dropped_while_a_stream_still_reads_it():
    net, _, _, x = model(14, 512, 1024, 2000, 2, 40)
    want = net(x)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
    got = net(x, stream=s)
    sizes = [t.numel() * t.element_size() for part in net.blocks + [net.head] for t in part._memory]
    del net
    taken = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(taken) == 3 * len(sizes)
