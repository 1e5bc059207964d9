"""Sequences that share a row of the page table."""
import pytest
import torch

from paper_2007_06919_gb300 import aqd
from test_gpu_lm_cache_attention import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,count", [(300, 5), (9000, 40)])
@pytest.mark.parametrize("dim", [64, 256])
def test_one_row_for_all(n, count, dim):
    c = Case([n], [1], 4, 2, dim, 16, torch.bfloat16, seed=30)
    q = torch.randn(count, 4, dim, device="cuda", dtype=torch.bfloat16)
    lengths = torch.linspace(1, n, count, device="cuda").int()
    want = aqd.cache_attention(q, c.cache, c.table.expand(count, -1).contiguous(), lengths)
    assert torch.equal(aqd.cache_attention(q, c.cache, c.table.expand(count, -1), lengths), want)
    wide = torch.cat([c.table, torch.full_like(c.table, -1)], 1)
    assert torch.equal(aqd.cache_attention(q[:1], c.cache, wide[:, :c.table.shape[1]], lengths[:1]), want[:1])
