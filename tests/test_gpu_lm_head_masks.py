"""The slope by the head's scales beside tokens, and places, that are masked: these add nothing, whatever their logits hold."""
import math

import pytest
import torch

from test_gpu_lm_decoder import model

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pad", [math.nan, math.inf, -math.inf])
def test_padded_tokens(pad):
    net, _, _, x = model(21, 128, 256, 300, 1, 24)
    head, logits = net.head, net(x)
    t = (logits.float() + torch.randn(24, 300, device="cuda", generator=torch.Generator("cuda").manual_seed(2))).topk(9)
    w = torch.ones(24, device="cuda")
    w[[3, 20]] = 0
    _, want = head.distill(logits, t.indices, t.values, tau=1.5, row_weight=w)
    x[[3, 20]] = pad
    padded = net(x)
    torch.cuda.synchronize()
    assert padded[[3, 20]].isnan().all()  # a row that holds a NaN or an infinity has no codes
    loss, got = head.distill(padded, t.indices, t.values, tau=1.5, row_weight=w, rate=0.1)
    assert (loss[[3, 20]] == 0).all() and torch.equal(got, want)
    assert head.proj.scales.isfinite().all() and (head.proj.scales > 0).all()


def test_masked_vocabulary():
    """Places that a mask rules out: q is 0 there, and so is what they add."""
    net, _, _, x = model(22, 128, 256, 300, 1, 24)
    logits = net(x)
    t = logits.float().mul(1.2)[:, :250].topk(9)
    logits[:, 250:] = -math.inf
    _, slope = net.head.distill(logits, t.indices, t.values)
    assert (slope[250:] == 0).all() and slope.isfinite().all() and (slope != 0).any()


def test_a_token_that_counts_and_is_not_finite_shows():
    net, _, _, x = model(23, 128, 256, 300, 1, 8)
    logits = net(x)
    t = logits.float().topk(9)
    logits[2, 5] = math.nan
    _, slope = net.head.distill(logits, t.indices, t.values)
    assert slope.isnan().all()
