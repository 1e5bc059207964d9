"""Distillation, further rows: tokens whose kept teacher logits hold a NaN or an infinity."""
import math

import pytest
import torch

from paper_2007_06919_gb300 import aqd
from test_gpu_lm_distill import TYPES, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("vocab", [50, 5001, 140000, 1700003])
@pytest.mark.parametrize("dtype", TYPES)
def test_a_token_without_a_teacher_distribution(vocab, dtype, bad):
    """p is not a number there, so q_v sum_j p_j is none at any v; the other tokens keep their values."""
    x, index, teacher, w = inputs(2, 6, vocab, 40, dtype)
    good = aqd.distill_topk(x, index, teacher, row_weight=w, grad=True)
    back = aqd.distill_topk_backward(x, index, teacher, good.lse, w)
    teacher[1, 0], teacher[4, 39] = bad, bad
    teacher[5, 7], index[5, 7] = bad, -1  # an empty place
    w[5] = 0
    out = aqd.distill_topk(x, index, teacher, row_weight=w, grad=True)
    again = aqd.distill_topk_backward(x, index, teacher, good.lse, w)
    torch.cuda.synchronize()
    assert torch.equal(out.lse, good.lse)
    for grad, before in ((out.grad, good.grad), (again, back)):
        assert grad[1].isnan().all() and grad[4].isnan().all() and (grad[5] == 0).all()
        for r in (0, 2, 3):
            assert torch.equal(grad[r], before[r])
    assert out.loss[1].isnan() and out.loss[4].isnan() and out.loss[5] == 0 and out.loss[[0, 2, 3]].isfinite().all()
