"""Keys alone of one head, wide and turned whole, of many tokens: blocks of many tokens keep a sine and a cosine for each pair of each."""
import pytest
import torch

from paper_2007_06919_gb300 import aqd
from test_gpu_lm_heads import freqs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,rot,dtype,pad", [(512, 512, torch.float32, 0), (512, 512, torch.bfloat16, 1), (512, 400, torch.float32, 0), (386, 386, torch.float16, 0)])
def test_many_keys_of_one_head(dim, rot, dtype, pad):
    n = 20_000
    torch.manual_seed(1)
    k = torch.randn(n, 1, dim + pad, device="cuda").to(dtype)[..., pad:]
    none = k[:, :0]
    w, pos, f = torch.ones(dim, device="cuda", dtype=dtype), torch.arange(n, device="cuda"), freqs(rot)
    got = aqd.qk_norm_rope(none, k, pos, f, k_weight=w).k
    parts = [aqd.qk_norm_rope(none[a:a + 500], k[a:a + 500], pos[a:a + 500], f, k_weight=w).k for a in range(0, n, 500)]
    assert torch.equal(got, torch.cat(parts))
