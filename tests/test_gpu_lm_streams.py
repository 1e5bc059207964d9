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
