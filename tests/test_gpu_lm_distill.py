"""aqd_distill_topk and its backward against the formulas in 64 bits, automatic differentiation of them, and differences.

Tolerances, with e = 2^-24 and z the largest |logit / tau| of the inputs (about 20): each z carries one rounding, its exponential
then z e and a few e; sums of float32 shares add (terms per thread + 16) e, at most 2^9 e here. So lse is within
(|lse| + 2 z + 600) e of its value, ln q and q's relative error likewise, the loss (a mean of ln p - ln q)
within 4 (z + |lse| + 600) e, and the gradient within that times (q + p) w / tau plus its type's own rounding."""
import math

import pytest
import torch

from paper_2007_06919_gb300 import aqd

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 1e-37, torch.float16: 2.0 ** -24, torch.bfloat16: 1e-37}
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def inputs(seed, tokens, vocab, top, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = (3 * torch.randn(tokens, vocab, generator=g, device="cuda")).to(dtype)
    t = (x.float() + torch.randn(tokens, vocab, generator=g, device="cuda")).topk(min(top, vocab), dim=1)
    index, teacher = t.indices, t.values.contiguous()
    if top > vocab:  # more places than the vocabulary has: the rest is empty
        index = torch.nn.functional.pad(index, (0, top - vocab), value=-1)
        teacher = torch.nn.functional.pad(teacher, (0, top - vocab))
    w = torch.rand(tokens, generator=g, device="cuda")
    return x, index, teacher, w


def plain(x, index, teacher, w, tau):
    """(loss, lse, q, p on the vocabulary) in 64 bits; x may require a gradient."""
    vocab = x.shape[1]
    z = x / tau
    lse = z.logsumexp(1)
    inside = (index >= 0) & (index < vocab)
    t = torch.where(inside, teacher.double() / tau, -math.inf)
    some = (t > -math.inf).any(1, keepdim=True)
    lp = torch.where(some, t, 0.0).log_softmax(1)
    p = torch.where(inside & (t > -math.inf), lp.exp(), 0.0)
    at = torch.where(inside, index, 0)
    lq = z.gather(1, at) - lse[:, None]
    term = torch.where(p > 0, p * (torch.where(p > 0, lp, 0.0) - torch.where(p > 0, lq, 0.0)), 0.0)
    wd = w.double() if w is not None else torch.ones(len(x), dtype=torch.float64, device=x.device)
    loss = torch.where(some.squeeze(1) & (wd != 0), wd * term.sum(1), 0.0)
    full = torch.zeros_like(x).scatter_add(1, at, p.to(x.dtype))
    return loss, lse, (z - lse[:, None]).exp(), full, some.squeeze(1)


def gradient(x, index, teacher, w, tau):
    _, _, q, full, some = plain(x.double(), index, teacher, w, tau)
    wd = w.double() if w is not None else torch.ones(len(x), dtype=torch.float64, device=x.device)
    f = torch.where(some, wd / tau, 0.0)[:, None]
    return f * (q - full), f * (q + full)


def check(x, index, teacher, w, tau):
    dtype = x.dtype
    loss, lse, _, _, _ = plain(x.double(), index, teacher, w, tau)
    grad, size = gradient(x, index, teacher, w, tau)
    z = (x.double().abs().max() / tau).item()
    wide = (z + lse.abs() + 600) * E
    factor = torch.ones_like(lse) if w is None else w.double()

    def near(got, what):
        torch.cuda.synchronize()
        off = (got.double() - grad).abs()
        allowed = 4 * wide[:, None] * size + HALF[dtype] * grad.abs() * 1.01 + TINY[dtype]
        assert (off <= allowed).all(), f"{what}: {(off - allowed).max().item()}"

    out = aqd.distill_topk(x, index, teacher, tau=tau, row_weight=w)
    torch.cuda.synchronize()
    assert out.grad is None
    assert ((out.lse.double() - lse).abs() <= 2 * wide).all()
    assert ((out.loss.double() - loss).abs() <= 4 * factor * wide).all()
    step = aqd.distill_topk(x, index, teacher, tau=tau, row_weight=w, grad=True)
    near(step.grad, "step")
    assert torch.equal(step.loss, out.loss) and torch.equal(step.lse, out.lse)
    near(aqd.distill_topk_backward(x, index, teacher, out.lse, w, tau=tau), "backward")
    again = aqd.distill_topk(x, index, teacher, tau=tau, row_weight=w, grad=True)
    torch.cuda.synchronize()
    assert torch.equal(again.grad, step.grad)  # a fixed order of sums


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 5, 31, 64, 1000, 1001, 4096, 8200, 32000, 32769, 50257, 65536, 131072, 131080, 200003, 600001])
def test_vocabularies(vocab, dtype):
    x, index, teacher, w = inputs(vocab, 3, vocab, 16, dtype)
    check(x, index, teacher, w, 1.0)
    check(x, index, teacher, None, 2.5)


@pytest.mark.parametrize("tokens", [1, 2, 19, 38, 76, 152, 153, 400])
def test_tokens(tokens):
    check(*inputs(tokens, tokens, 16000, 8, torch.bfloat16), 1.0)


@pytest.mark.parametrize("top", [1, 2, 33, 64, 257, 512, 1000, 1024])
def test_kept_places(top):
    check(*inputs(top, 5, 2000, top, torch.float32), 1.5)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("start,pad", [(0, 8), (1, 0), (3, 5), (8, 1), (0, 1)])
def test_strides_addresses_and_in_place(start, pad, dtype):
    tokens, vocab = 7, 5000
    x0, index, teacher, w = inputs(4, tokens, vocab, 9, dtype)
    whole = torch.full((tokens, start + vocab + pad), 7.0, dtype=dtype, device="cuda")
    x = whole[:, start:start + vocab]
    x.copy_(x0)
    check(x, index, teacher, w, 1.0)
    want = aqd.distill_topk(x0, index, teacher, row_weight=w, grad=True)
    other = torch.full((tokens, vocab + 16), 7.0, dtype=dtype, device="cuda")
    got = aqd.distill_topk(x, index, teacher, row_weight=w, grad=other[:, 3:3 + vocab])
    torch.cuda.synchronize()
    assert (other[:, :3] == 7).all() and (other[:, 3 + vocab:] == 7).all()
    allowed = 8 * (20 + 600) * E
    assert ((got.grad.float() - want.grad.float()).abs() <= allowed + 2 * HALF[dtype] * want.grad.float().abs() + TINY[dtype]).all()
    lse = got.lse.clone()
    kept = got.grad.clone()
    aqd.distill_topk(x, index, teacher, row_weight=w, grad=x)
    torch.cuda.synchronize()
    assert torch.equal(x, kept)
    x.copy_(x0)
    aqd.distill_topk_backward(x, index, teacher, lse, w, grad=x)
    torch.cuda.synchronize()
    near = (x.float() - kept.float()).abs() <= allowed + 2 * HALF[dtype] * kept.float().abs() + TINY[dtype]
    assert near.all()
    assert (whole[:, :start] == 7).all() and (whole[:, start + vocab:] == 7).all()


@pytest.mark.parametrize("vocab", [40, 3001, 140000])
def test_masked_logits_empty_and_repeated_places(vocab):
    x, index, teacher, w = inputs(1, 8, vocab, 12, torch.float32)
    w[:] = 0.5
    index[0, 3:] = -1                    # fewer kept logits
    index[1] = -1                        # none
    index[2, 5] = vocab                  # past the vocabulary
    index[3] = index[3, 0]               # one place twelve times
    teacher[4, 2:] = -math.inf
    teacher[5] = -math.inf               # none
    teacher[1, 2] = math.nan             # in an empty place
    low = torch.full_like(x, -math.inf)  # a vocabulary masked down to the kept places
    x[6] = low[6].scatter(0, index[6], x[6].gather(0, index[6]))
    x[7] = torch.where(torch.arange(vocab, device="cuda") % 2 == 0, torch.finfo(torch.float32).min, x[7])
    x[7].scatter_(0, index[7], 1.0)
    t2 = teacher.clone()
    t2[1, 2] = 0.0
    loss, lse, _, _, _ = plain(x.double(), index, t2, w, 1.0)
    grad, size = gradient(x, index, t2, w, 1.0)
    out = aqd.distill_topk(x, index, teacher, row_weight=w, grad=True)
    back = aqd.distill_topk_backward(x, index, teacher, out.lse, w)
    torch.cuda.synchronize()
    assert out.loss[1] == 0 and out.loss[5] == 0 and (out.grad[1] == 0).all() and (out.grad[5] == 0).all()
    wide = (40 + lse.abs() + 600) * E
    assert ((out.lse.double() - lse).abs() <= 2 * wide).all()
    assert ((out.loss.double() - loss).abs() <= 4 * wide).all()
    for g in (out.grad, back):
        assert ((g.double() - grad).abs() <= 4 * wide[:, None] * size + 1e-37).all()


@pytest.mark.parametrize("vocab", [50, 5001, 140000])
@pytest.mark.parametrize("dtype", TYPES)
def test_weight_zero_and_non_finite_rows(vocab, dtype):
    x, index, teacher, w = inputs(2, 8, vocab, 6, dtype)
    w[:] = 1
    w[0] = 0
    x[0] = math.nan                      # a padded token
    x[1, vocab // 2] = math.nan
    x[2, vocab - 1] = math.inf
    x[3] = -math.inf
    x[4, index[4, 1]] = -math.inf        # a kept place that the student rules out
    teacher[5, 2] = math.nan
    teacher[6, 0] = math.inf
    out = aqd.distill_topk(x, index, teacher, row_weight=w, grad=True)
    back = aqd.distill_topk_backward(x, index, teacher, out.lse, w)
    torch.cuda.synchronize()
    assert out.loss[0] == 0 and (out.grad[0] == 0).all() and (back[0] == 0).all()
    for r in (1, 2, 3, 5, 6):
        assert out.loss[r].isnan(), r
    for r in (1, 2, 3):
        assert out.grad[r].isnan().all() and back[r].isnan().all(), r
    for r in (5, 6):
        assert out.grad[r].isnan().any() and back[r].isnan().any(), r
    assert out.loss[4] == math.inf and out.grad[4].isfinite().all() and out.grad[4, index[4, 1]] < 0
    assert out.loss[7].isfinite() and out.grad[7].isfinite().all()


@pytest.mark.parametrize("vocab", [50, 5001, 140000])
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_the_lowest_value(vocab, dtype):
    """Every z - m is 0 then, exactly: q is even, and what rounds are the sums, logarithms and exponentials."""
    x, index, teacher, w = inputs(3, 3, vocab, 6, dtype)
    w[:] = 1
    x[0] = torch.finfo(dtype).min                    # no logit left by a mask
    teacher[1] = torch.finfo(torch.float32).min      # the teacher's kept logits alike
    x[2] = torch.finfo(dtype).min
    teacher[2, 1:] = torch.finfo(torch.float32).min  # one kept logit
    out = aqd.distill_topk(x, index, teacher, row_weight=w, grad=True)
    # less each row's maximum, which changes neither loss nor gradient: ln V is lost beside 3e38 in 64 bits too
    shifted = x.double() - x.double().amax(1, keepdim=True)
    loss, _, _, _, _ = plain(shifted, index, teacher, w, 1.0)
    grad, size = gradient(shifted, index, teacher, w, 1.0)
    torch.cuda.synchronize()
    wide = (20 + math.log(vocab) + 600) * E
    assert ((out.loss.double() - loss).abs() <= 4 * wide).all()
    assert ((out.grad.double() - grad).abs() <= 4 * wide * size + HALF[dtype] * grad.abs() * 1.01 + TINY[dtype]).all()


def test_gradient_of_the_formula_and_differences():
    x, index, teacher, w = inputs(9, 4, 300, 10, torch.float32)
    index[0, 4] = index[0, 1]
    index[1, 7] = -1
    tau = 1.7
    got = aqd.distill_topk(x, index, teacher, tau=tau, row_weight=w, grad=True).grad.double()
    xd = x.double().requires_grad_()
    plain(xd, index, teacher, w, tau)[0].sum().backward()
    z = 20
    allowed = 4 * (z + 30 + 600) * E
    assert ((got - xd.grad).abs() <= allowed).all()
    # central differences of the loss in 64 bits: an error of h^2 / 6 times a third derivative below 1 / tau^3
    h = 1e-4
    places = torch.cat([index[:, :3].clamp(min=0), torch.tensor([[0, 17, 299]] * 4, device="cuda")], 1)
    for j in range(places.shape[1]):
        step = torch.zeros_like(xd).scatter(1, places[:, j:j + 1], h)
        d = (plain(x.double() + step, index, teacher, w, tau)[0] - plain(x.double() - step, index, teacher, w, tau)[0]) / (2 * h)
        assert ((got.gather(1, places[:, j:j + 1]).squeeze(1) - d).abs() <= allowed + 1e-8).all()


def test_offsets_past_32_bits():
    tokens, vocab, ld = 4, 1000, 900_000_001
    x0, index, teacher, w = inputs(5, tokens, vocab, 8, torch.bfloat16)
    x = torch.empty((tokens - 1) * ld + vocab, dtype=torch.bfloat16, device="cuda").as_strided((tokens, vocab), (ld, 1))
    x.copy_(x0)
    check(x, index, teacher, w, 1.0)
    aqd.distill_topk(x, index, teacher, row_weight=w, grad=x)
    want = gradient(x0, index, teacher, w, 1.0)[0]
    assert ((x.double() - want).abs() <= HALF[torch.bfloat16] * want.abs() * 1.01 + 1e-4).all()


def test_leading_dimensions_no_tokens_streams_and_graphs():
    x, index, teacher, w = inputs(6, 12, 700, 5, torch.float16)
    want = aqd.distill_topk(x, index, teacher, row_weight=w, grad=True)
    got = aqd.distill_topk(x.view(3, 4, 700), index.view(3, 4, 5), teacher.view(3, 4, 5), row_weight=w.view(3, 4), grad=True)
    torch.cuda.synchronize()
    assert got.loss.shape == (3, 4) and torch.equal(got.loss.view(-1), want.loss) and torch.equal(got.grad.view(12, 700), want.grad)
    none = aqd.distill_topk(x[:0], index[:0], teacher[:0], grad=True)
    assert none.loss.shape == (0,) and none.grad.shape == (0, 700)
    s = torch.cuda.Stream()
    other = aqd.distill_topk(x, index, teacher, row_weight=w, grad=True, stream=s)
    s.synchronize()
    assert torch.equal(other.grad, want.grad)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = aqd.distill_topk(x, index, teacher, row_weight=w, grad=True)
    y.grad.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y.grad, want.grad) and torch.equal(y.loss, want.loss)


def test_refusals():
    x, index, teacher, w = inputs(6, 12, 700, 5, torch.float16)
    bad = [lambda: aqd.distill_topk(x.int(), index, teacher), lambda: aqd.distill_topk(x, index.int(), teacher),
           lambda: aqd.distill_topk(x, index, teacher.half()), lambda: aqd.distill_topk(x, index[:, :4], teacher),
           lambda: aqd.distill_topk(x[:6], index, teacher), lambda: aqd.distill_topk(x, index, teacher, row_weight=w[:3]),
           lambda: aqd.distill_topk(x, index, teacher, grad=x.float()), lambda: aqd.distill_topk(x.t(), index, teacher),
           lambda: aqd.distill_topk_backward(x, index, teacher, w[:3]), lambda: aqd.distill_topk(x.cpu(), index, teacher)]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for tau in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(aqd.AqdError):
            aqd.distill_topk(x, index, teacher, tau=tau)
    many = torch.zeros(12, 1025, dtype=torch.int64, device="cuda")
    with pytest.raises(aqd.AqdError):
        aqd.distill_topk(x, many, many.float())
    with pytest.raises(aqd.AqdError):
        aqd.distill_topk(x, index[:, :0].contiguous(), teacher[:, :0].contiguous())
    with pytest.raises(aqd.AqdError):  # rows of the gradient that overlap
        aqd.distill_topk(x, index, teacher, grad=x[:1].expand(12, 700))
