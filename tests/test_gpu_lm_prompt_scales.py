"""Attention over packed prompts with scales that float32 can just hold."""
import pytest
import torch

from attention_ref import close
from paper_2007_06919_gb300 import aqd
from test_gpu_lm_prompt import inputs, reference, starts_of

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def laid_out(q, layout):
    """Queries as they are, or one head's for all of them (a stride of zero: the kernel without a tensor map)."""
    return q if layout == "own" else q[:, :1].expand(q.shape)


def run(q, k, v, starts, **more):
    return aqd.prompt_attention(q, k, v, starts, out=torch.empty(q.shape, device="cuda", dtype=q.dtype), lse=True, **more)


LAYOUTS = ["own", "broadcast"]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dim", [64, 128, 192, 256])
@pytest.mark.parametrize("scale", [1e-39, 1e-38, 1.7e-38, 1e-30])
def test_a_scale_that_leaves_no_difference(dim, scale, layout):
    at, starts = starts_of([200, 1, 300])
    q, k, v = inputs(dim, at[-1], at[-1], 2, 1, dim, BF16)
    q = laid_out(q, layout)
    scale = torch.tensor(scale).item()
    o, tol, e, et = reference(q, k, v, at, at, True, scale)
    got, lse = run(q, k, v, starts, scale=scale)
    close(got, o, tol)
    close(lse, e, et)
