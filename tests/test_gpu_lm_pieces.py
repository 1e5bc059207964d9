"""More rows than a grid's second dimension has (65,535): calls are launched in pieces, every tensor's address moved on by hand. Rows on both sides of
a piece's end against calls of their own on the same memory, which take the same kernels in the same order of sums (that depends on where in its 16 bytes a
row starts): bit for bit."""
import pytest
import torch

from paper_2007_06919_gb300 import aqd
from test_gpu_lm_distill import inputs
from test_gpu_lm_linear import codes, scaled, scales, sums

pytestmark = pytest.mark.gpu

END = 65535


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens", [END + 65, 2 * END + 3])
def test_distillation(tokens, dtype):
    x, index, teacher, w = inputs(1, tokens, 203, 7, dtype)
    out = aqd.distill_topk(x, index, teacher, tau=1.5, row_weight=w, grad=True)
    loss = aqd.distill_topk(x, index, teacher, tau=1.5, row_weight=w)
    back = aqd.distill_topk_backward(x, index, teacher, out.lse, w, tau=1.5)
    even = aqd.distill_topk(x, index, teacher, tau=1.5)
    torch.cuda.synchronize()
    assert torch.equal(loss.loss, out.loss) and torch.equal(loss.lse, out.lse)
    # (the last token, and the second piece's end, are among them)
    for lo in (0, END - 40, tokens - 60):
        at = slice(lo, lo + 60)
        a, i, t = x[at], index[at], teacher[at]
        want = aqd.distill_topk(a, i, t, tau=1.5, row_weight=w[at], grad=True)
        grad = aqd.distill_topk_backward(a, i, t, want.lse, w[at], tau=1.5)
        alone = aqd.distill_topk(a, i, t, tau=1.5)
        torch.cuda.synchronize()
        assert torch.equal(out.loss[at], want.loss) and torch.equal(out.lse[at], want.lse) and torch.equal(out.grad[at], want.grad)
        assert torch.equal(back[at], grad) and torch.equal(even.loss[at], alone.loss)


@pytest.mark.parametrize("values", [False, True])
def test_rows_in_clusters(values):
    """(at least 304 rows in the calls of their own, which then take as many blocks a row)"""
    rows, cols, dtype = END + 70, 18440, torch.bfloat16
    g = torch.Generator("cuda").manual_seed(3)
    x, r = (torch.empty(rows, cols, dtype=dtype, device="cuda").normal_(generator=g) for _ in range(2))
    w = 1 + 0.3 * torch.randn(cols, device="cuda", generator=g)
    q = aqd.rms_norm_quant(x, w, residual=r, values=values)
    gate = aqd.gated_act_quant(x, r, codes=not values, values=values)
    torch.cuda.synchronize()
    for lo in (0, END - 200, rows - 310):
        at = slice(lo, lo + 310)
        a, b = x[at], r[at]
        for got, want in ((q, aqd.rms_norm_quant(a, w, residual=b, values=values)), (gate, aqd.gated_act_quant(a, b, codes=not values, values=values))):
            for u, v in zip(got, want):
                assert (u is None and v is None) or torch.equal(u[at], v)
    in_place = aqd.rms_norm_quant(x, w, residual=r, summed=x)
    torch.cuda.synchronize()
    assert torch.equal(x, q.summed) and torch.equal(in_place.codes, q.codes) and torch.equal(in_place.scales, q.scales)


@pytest.mark.parametrize("pad", [0, 1])
def test_products_without_a_workspace(pad):
    """64 tokens a block, or 32 at any address."""
    step = 64 if pad == 0 else 32
    m, k, n = step * END + 77, 16, 9
    wc, xs = codes(2, n, k), scales(3, m)
    layer = aqd.LinearWeights(wc, scales(4, n))
    x = codes(1, m, k + pad)[:, :k]
    got = aqd.linear_int8(x, xs, layer, out_dtype=torch.float32)
    ints = aqd.linear_int8(x, None, layer, out_dtype=torch.int32)
    torch.cuda.synchronize()
    s = sums(x, wc)
    assert torch.equal(ints, s.int()) and torch.equal(got, scaled(s, xs, layer.scales, None, torch.float32))
