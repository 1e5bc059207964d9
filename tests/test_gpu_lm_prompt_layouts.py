"""Attention over packed prompts where strides are zero (the kernel without a tensor map), and with more sequences than a grid's second axis has blocks."""
import math

import pytest
import torch

from attention_ref import close
from paper_2007_06919_gb300 import aqd
from test_gpu_lm_prompt import LENS, inputs, reference, starts_of
from test_gpu_lm_prompt_scales import run

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def one_for_all(q, k, v, which):
    """One head's rows for all heads, or one token's for all tokens."""
    if which == "queries":
        return q[:, :1].expand(q.shape), k, v
    if which == "keys":
        return q, k[:, :1].expand(k.shape), v
    if which == "values":
        return q, k, v[:, :1].expand(v.shape)
    return q[:1].expand(q.shape), k, v


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("which,heads,kv,dim,dtype", [("queries", 4, 2, 64, BF16), ("keys", 4, 2, 128, F16), ("values", 2, 2, 192, BF16), ("tokens", 6, 1, 256, F16),
                                                      ("tokens", 3, 3, 64, F16), ("queries", 2, 1, 128, BF16), ("keys", 4, 2, 192, F16), ("values", 4, 2, 256, BF16)])
def test_packed_prompts(which, heads, kv, dim, dtype, causal):
    at, starts = starts_of(LENS)
    q, k, v = one_for_all(*inputs(dim + heads, at[-1], at[-1], heads, kv, dim, dtype), which)
    o, tol, e, et = reference(q, k, v, at, at, causal, dim ** -0.5)
    got, lse = run(q, k, v, starts, causal=causal)
    close(got, o, tol)
    close(lse, e, et)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("which,dim,dtype", [("queries", 128, BF16), ("keys", 64, F16), ("values", 192, F16), ("tokens", 256, BF16)])
def test_other_keys_than_queries(which, dim, dtype, causal):
    lens, klens = [5, 100, 1, 64, 0, 40, 7, 300], [500, 100, 700, 10, 30, 0, 7, 40]
    at, starts = starts_of(lens)
    kat, kstarts = starts_of(klens)
    q, k, v = one_for_all(*inputs(dim, at[-1], kat[-1], 4, 2, dim, dtype), which)
    o, tol, e, et = reference(q, k, v, at, kat, causal, 0.2)
    got, lse = run(q, k, v, starts, kv_starts=kstarts, causal=causal, scale=0.2)
    close(got, o, tol)
    close(lse, e, et)
    assert (got[at[5]:at[6]] == 0).all() and (lse[at[5]:at[6]] == -math.inf).all()


@pytest.mark.parametrize("dim", [64, 192])
def test_sequences_around_the_second_axis(dim):
    """Sequences of a token or none, a few units below and above 65,535 of them: a token sees itself alone, so its output is its value."""
    rows = 256 if dim == 64 else 128
    for over in (-1, 0, 1, 70):
        tokens = 60_000
        seqs = 65_535 - tokens // rows + over
        torch.manual_seed(dim)
        lens = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        lens[torch.randperm(seqs, device="cuda")[:tokens]] = 1
        starts = torch.cat([lens.new_zeros(1), lens.cumsum(0, dtype=torch.int32)])
        q, k, v = (torch.randn(tokens, 2 if i == 0 else 1, dim, device="cuda", dtype=BF16) for i in range(3))
        got, lse = run(q, k, v, starts, scale=0.125)
        assert torch.equal(got, v.expand(-1, 2, -1))
        want = 0.125 * torch.einsum("thd,tkd->th", q.double(), k.double())
        # a sum of dim products in float32, cut at 2^-22 of the largest partial sum for each of dim / 16 steps
        size = 0.125 * torch.einsum("thd,tkd->th", q.double().abs(), k.double().abs())
        close(lse, want, size * (dim / 16 + 6) * 2.0 ** -22 + 2.0 ** -21)
    assert aqd.device_status() == 0
