"""The decoder's 8-bit feed-forward blocks, head and distillation, the operators run together as a program runs them."""
import pytest
import torch

from paper_2007_06919_gb300 import aqd
from paper_2007_06919_gb300.feedforward import Decoder, FeedForward, Head

pytestmark = pytest.mark.gpu


def model(seed, d, hidden, vocab, layers, tokens, act="silu", dtype=torch.bfloat16):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    w = [((1 + 0.1 * normal(d)).to(dtype), normal(hidden, d) / d ** 0.5, normal(hidden, d) / d ** 0.5, normal(d, hidden) / hidden ** 0.5)
         for _ in range(layers)]
    hn, hw = (1 + 0.1 * normal(d)).to(dtype), 2 * normal(vocab, d) / d ** 0.5
    net = Decoder([FeedForward(*b, act=act, tokens=tokens) for b in w], Head(hn, hw, tokens=tokens))
    return net, w, (hn, hw), normal(tokens, d).to(dtype)


def plain(w, head, x, act):
    """The float model in 64 bits."""
    def norm(t, weight):
        return t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6) * weight.double()

    y, r = x.double(), torch.zeros_like(x, dtype=torch.float64)
    for nw, gate, up, down in w:
        r = r + y
        h = norm(r, nw)
        a = h @ gate.double().T
        a = torch.nn.functional.silu(a) if act == "silu" else torch.nn.functional.gelu(a, approximate="tanh")
        y = (a * (h @ up.double().T)) @ down.double().T
    return norm(r + y, head[0]) @ head[1].double().T


# A code's rounding is s / sqrt(12) with s = max / 127: 0.8% of normal rows (maximum 3.5 deviations), 2 to 3% of the gated
# products (maximum 10). A block adds about 1.1% from its first products (1.6% past the gate), 2.5% from the codes after, 0.8% from the
# down weights, 16-bit roundings of 0.3%: 3.2% of its output, half of the sum's square; two blocks and the head stay below 5%.
@pytest.mark.parametrize("d,hidden,vocab,tokens,act", [(256, 512, 1000, 1, "silu"), (512, 1024, 2000, 24, "gelu_tanh"), (130, 257, 999, 77, "silu"),
                                                     (1024, 2048, 4096, 512, "silu")])
def test_forward_against_the_float_model(d, hidden, vocab, tokens, act):
    net, w, head, x = model(d, d, hidden, vocab, 2, tokens, act)
    got, want = net(x).double(), plain(w, head, x, act)
    assert got.shape == (tokens, vocab)
    assert (got - want).norm() <= 0.08 * want.norm()


@pytest.mark.parametrize("tokens", [1, 16, 40, 300])
def test_forward_is_its_operators_in_sequence_and_each_token_alone(tokens):
    net, _, _, x = model(3, 256, 512, 1000, 2, tokens)
    logits = net(x)
    y, r = x, None
    for b in net.blocks:
        q = aqd.rms_norm_quant(y, b.norm, eps=b.eps, residual=r)
        both = aqd.linear_int8(q.codes, q.scales, b.both)
        h = aqd.gated_act_quant(both[:, :b.hidden].contiguous(), both[:, b.hidden:].contiguous(), act=b.act)
        r = y if r is None else q.summed
        y = aqd.linear_int8(h.codes, h.scales, b.down)
    q = aqd.rms_norm_quant(y, net.head.norm, residual=r)
    assert torch.equal(logits, aqd.linear_int8(q.codes, q.scales, net.head.proj))
    # exact sums and scales of a token's own: a token's logits do not depend on the others
    at = tokens // 2
    assert torch.equal(net(x[at:at + 1])[0], logits[at])
    assert torch.equal(net(x.view(1, tokens, -1))[0], logits)


def test_scale_gradient_and_steps():
    net, _, _, x = model(5, 128, 256, 300, 1, 64)
    head = net.head
    logits = net(x)
    t = (logits.float() * 1.3 + torch.randn(64, 300, device="cuda", generator=torch.Generator("cuda").manual_seed(1))).topk(12)
    _, slope = head.distill(logits, t.indices, t.values, tau=1.5)
    # the same loss in 64 bits, by the logarithms of factors of the logits
    f = torch.zeros(300, dtype=torch.float64, device="cuda", requires_grad=True)

    def loss(by):
        lq = (logits.double() * by.exp() / 1.5).log_softmax(1).gather(1, t.indices)
        lp = (t.values.double() / 1.5).log_softmax(1)
        return (lp.exp() * (lp - lq)).sum()

    loss(f).backward()
    # bfloat16 gradients, 2^-9 of each entry's size, and the float32 terms' sums
    size = ((logits.double() / 1.5).softmax(1) + 1).mul(logits.double().abs() / 1.5).sum(0)
    assert ((slope.double() - f.grad).abs() <= 2 ** -8 * size).all()
    with torch.no_grad():
        h = 1e-4
        for v in (0, 17, int(t.indices[0, 0])):
            e = torch.zeros_like(f)
            e[v] = h
            assert abs((loss(e) - loss(-e)).item() / (2 * h) - f.grad[v].item()) <= 1e-5 * (1 + size[v].item())
    first = None
    for _ in range(20):
        out, _ = head.distill(net(x), t.indices, t.values, tau=1.5, rate=0.05)
        first = out.mean() if first is None else first
    assert (head.proj.scales > 0).all() and out.mean() < first


def test_streams_graphs_and_refusals():
    net, w, _, x = model(7, 256, 512, 1000, 2, 40)
    want = net(x)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = net(x, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    static = x.clone()
    with torch.cuda.graph(g):
        y = net(static)
    y.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    static.copy_(x.flip(0))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, want.flip(0))
    norm, gate, up, down = w[0]
    for bad in ((norm, gate, up[:5], down), (norm, gate, up, gate), (norm[:5], gate, up, down)):
        with pytest.raises(ValueError):
            FeedForward(*bad)
    with pytest.raises(ValueError):
        net(x[:, :200])
