"""Attention with the largest scales: each query takes the value of its best key alone."""
import pytest
import torch

from paper_2007_06919_gb300 import aqd
from test_gpu_lm_prompt_scales import LAYOUTS, laid_out, run

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dim,dtype", [(64, BF16), (128, F16), (192, BF16), (256, F16)])
@pytest.mark.parametrize("scale", [1e30, 2.5e38, 3.4e38])
def test_prompts(dim, dtype, scale, layout):
    """Keys whose scores grow along the prompt, and ones whose scores fall: the last key seen, and the first."""
    n = 250
    torch.manual_seed(dim)
    v = torch.randn(2 * n, 2, dim, device="cuda").to(dtype)
    k = torch.zeros(2 * n, 2, dim, device="cuda", dtype=dtype)
    k[:n, :, 3] = torch.arange(n, device="cuda").to(dtype)[:, None]
    k[n:, :, 3] = -torch.arange(n, device="cuda").to(dtype)[:, None]
    q = torch.zeros(2 * n, 4, dim, device="cuda", dtype=dtype)
    q[..., 3] = 1
    starts = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
    got, _ = run(laid_out(q, layout), k, v, starts, scale=torch.tensor(scale).item())
    best = torch.cat([torch.arange(n), torch.full((n,), n)]).cuda()
    assert torch.equal(got, v[best].repeat_interleave(2, 1))


@pytest.mark.parametrize("dim,kv", [(64, 1), (128, 2), (256, 1)])
@pytest.mark.parametrize("scale,size", [(3.4e38, 1.0), (1e30, 1e4), (3.4e38, 2.0 ** 15), (1e20, 2.0 ** 100)])
def test_cache(dim, kv, scale, size):
    """Keys of one value, 15 times a power of two, and zeros: held exactly."""
    torch.manual_seed(dim)
    n = 40
    order = torch.randperm(n, device="cuda")
    k = torch.zeros(n, kv, dim, device="cuda")
    k[:, :, 5] = (15 * 2.0 ** (order.float() - 20))[:, None]
    v = torch.randn(n, kv, dim, device="cuda")
    cache = aqd.KVCache(3, 16, kv, dim)
    slots = torch.arange(n, device="cuda")
    aqd.cache_write(cache, k, v, slots)
    held = aqd.cache_read(cache, slots, dtype=torch.float32)[1]
    q = torch.zeros(1, 2 * kv, dim, device="cuda", dtype=BF16)
    q[..., 5] = size
    table, length = torch.arange(3, dtype=torch.int32, device="cuda")[None], torch.tensor([n], dtype=torch.int32, device="cuda")
    got = aqd.cache_attention(q, cache, table, length, scale=torch.tensor(scale).item())
    want = held[order.argmax()].repeat_interleave(2, 0)[None].double()
    # (a weight of 1 times the step, in float16, and times codes of up to 8 of it; the output's rounding)
    step = (held.amax(-1) - held.amin(-1)).max().item() / 15
    assert ((got.double() - want).abs() <= 2.0 ** -11 * 8.2 * step + 2.0 ** -8 * want.abs()).all()
