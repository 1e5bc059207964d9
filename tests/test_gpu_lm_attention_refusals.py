"""What the decoder's attention blocks refuse, before any cache is written."""
import pytest
import torch

from paper_2007_06919_gb300 import aqd
from paper_2007_06919_gb300.attention import Sequences
from test_gpu_lm_attention_decoder import model

pytestmark = pytest.mark.gpu


def test_types_that_attention_does_not_take_write_nothing():
    net, _, _, _ = model(9, 256, 512, 1000, 4, 2, 64, 2)
    seqs, caches = Sequences(20, 16, 8), net.caches(20, 16)
    for c in caches:
        c.data.fill_(0xA5)
    seqs.add(0)
    tokens = seqs.extend([0], [20])
    x = torch.randn(20, 256, device="cuda")
    with pytest.raises(ValueError, match="float16 or bfloat16"):
        net(x, tokens, caches)
    with pytest.raises(ValueError, match="float16 or bfloat16"):
        net.blocks[0][0](x, None, tokens, caches[0])
    with pytest.raises(ValueError, match="cache"):
        net(x.bfloat16(), tokens, caches[:1])
    with pytest.raises(ValueError, match="cache"):
        net(x.bfloat16(), tokens, caches + caches[:1])
    with pytest.raises(ValueError, match="cache"):
        net(x.bfloat16(), tokens, [caches[0], aqd.KVCache(20, 16, 1, 64)])
    assert all((c.data == 0xA5).all() for c in caches)
    net(x.bfloat16(), tokens, caches)
