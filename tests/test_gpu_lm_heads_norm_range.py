"""Norms of heads whose squares, or the sum of them, lie outside float32's range: their normalized values are ordinary ones. Compared as the other rows are, with
the formula in 64 bits."""
import math

import pytest
import torch

from attention_ref import close, rotated
from paper_2007_06919_gb300 import aqd
from test_gpu_lm_heads import bound, freqs

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

# a row's size, times values of up to 3: the largest below 3.4e38
SIZES = [1.0, 1e-12, 3e-18, 1e-19, 3e-20, 1e-20, 1e-21, 1e-22, 1e-23, 1e-27, 1e-32, 1e-37, 3e-39, 1e4, 1e17, 1e18, 2e18, 1e19, 3e19, 1e20, 1e27, 1e35, 1e38]


def rows(seed, heads, dim, dtype, pad):
    torch.manual_seed(seed)
    x = torch.randn(len(SIZES), heads, dim, device="cuda", dtype=torch.float64).clamp(-3, 3) * torch.tensor(SIZES, dtype=torch.float64, device="cuda")[:, None, None]
    both = torch.zeros(len(SIZES), heads * dim + pad, device="cuda", dtype=dtype)
    both[:, pad:] = x.to(dtype).flatten(1)
    return both[:, pad:].unflatten(1, (heads, dim))


@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-40, 2e-38, 1e-30, 1e-6])
@pytest.mark.parametrize("dtype,dim,rot,interleaved,pad", [
    (BF16, 128, 128, False, 0), (BF16, 64, 32, True, 0), (F32, 128, 0, False, 0), (F32, 256, 64, False, 0), (BF16, 512, 512, False, 0), (BF16, 192, 192, True, 0),
    (BF16, 128, 128, False, 1), (F32, 64, 64, True, 1), (F32, 512, 512, False, 0), (F32, 6, 2, False, 0)])
def test_rows_of_any_size(dtype, dim, rot, interleaved, pad, eps):
    eps = torch.tensor(eps).item()  # as float32 has it
    q, k = rows(dim, 3, dim, dtype, pad), rows(dim + 1, 2, dim, dtype, pad)
    w = (1 + 0.3 * torch.randn(dim, device="cuda")).to(dtype)
    pos, f = torch.arange(len(SIZES), device="cuda") * 1001, freqs(rot) if rot else None
    out = aqd.qk_norm_rope(q, k, pos, f, q_weight=w, k_weight=w, eps=eps, interleaved=interleaved)
    for x, got in ((q, out.q), (k, out.k)):
        want, size = rotated(x, w, pos, f, interleaved, eps)
        close(got, want, bound(want, size, dtype))


@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_to_the_cache_in_the_same_pass(dtype, pad):
    n = len(SIZES)
    q, k, v = rows(1, 2, 128, dtype, pad), rows(2, 2, 128, dtype, pad), rows(3, 2, 128, dtype, pad)
    w = (1 + 0.3 * torch.randn(128, device="cuda")).to(dtype)
    pos, f, slots = torch.arange(n, device="cuda"), freqs(128), torch.arange(n, device="cuda")
    one, two = (aqd.KVCache(2, 16, 2, 128) for _ in range(2))
    one.data.zero_(), two.data.zero_()
    want = aqd.qk_norm_rope(q, k, pos, f, q_weight=w, k_weight=w, eps=0.0)
    aqd.cache_write(two, want.k, v, slots)
    got = aqd.qk_norm_rope(q, k, pos, f, q_weight=w, k_weight=w, eps=0.0, v=v, cache=one, slots=slots)
    assert torch.equal(got.q, want.q) and torch.equal(one.data, two.data) and want.k.isfinite().all() and (want.k != 0).any(-1).all()


@pytest.mark.parametrize("dim", [64, 6, 512])
def test_one_value_and_special_rows(dim):
    """A single value in a row of zeros, beside rows that hold a NaN, an infinity, nothing but zeros: each row by its own values."""
    x = torch.zeros(8, 4, dim, device="cuda")
    x[0, 0, dim // 2], x[0, 1, 0], x[0, 2, dim - 1], x[0, 3, 1] = 1e-30, -1e-22, 3e-45, 3e38
    x[1, 0, 1], x[1, 1, 1], x[1, 3] = math.nan, math.inf, 1e-25
    x[2:] = torch.randn(6, 4, dim, device="cuda")
    w = torch.ones(dim, device="cuda")
    got = aqd.qk_norm_rope(x, x[:, :1].contiguous(), None, None, q_weight=w, eps=0.0).q
    want, size = rotated(x, w, None, None, False, 0.0)
    for t, h in ((0, slice(0, 4)), (1, slice(3, 4)), (slice(2, 8), slice(0, 4))):
        close(got[t, h], want[t, h], bound(want[t, h], size[t, h], F32))
    assert got[1, 0].isnan().all() and got[1, 1, 1].isnan() and got[1, 2].isnan().all()  # (zeros: 0 / 0)
    tiny = aqd.qk_norm_rope(x, x[:, :1].contiguous(), None, None, q_weight=w, eps=1e-6).q
    assert (tiny[1, 2] == 0).all()
