"""Attention over packed prompts: values that the causal order hides hold a NaN or an infinity."""
import math

import pytest
import torch

from attention_ref import close
from paper_2007_06919_gb300 import aqd
from test_gpu_lm_prompt import inputs, reference, starts_of
from test_gpu_lm_prompt_scales import LAYOUTS, laid_out, run

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("heads,kv,dim,dtype", [(4, 2, 64, F16), (2, 1, 128, BF16), (2, 2, 192, F16), (2, 1, 256, BF16), (2, 1, 64, BF16), (2, 2, 128, F16)])
def test_values_behind_a_query(heads, kv, dim, dtype, bad, layout):
    """Each of some places has one bad channel: queries before it are as if it were not there, the others have that channel alone spoiled."""
    lens = [700, 1, 200, 129, 40]
    at, starts = starts_of(lens)
    q, k, v = inputs(dim + heads, at[-1], at[-1], heads, kv, dim, dtype)
    q = laid_out(q, layout)
    o, tol, e, et = reference(q, k, v, at, at, True, dim ** -0.5)
    vv, spoiled = v.clone(), torch.zeros(at[-1], heads, dim, dtype=torch.bool, device="cuda")
    for s, places in ((0, (3, 63, 64, 127, 128, 129, 255, 256, 300, 511, 640, 699)), (1, (0,)), (2, (0, 130, 199)), (3, (127, 128))):
        for i, t in enumerate(places):
            c, h = (17 * i + 5) % dim, i % kv
            vv[at[s] + t, h, c] = bad
            spoiled[at[s] + t:at[s + 1], h * (heads // kv):(h + 1) * (heads // kv), c] = True
    got, lse = run(q, k, vv, starts)
    assert not got[spoiled].isfinite().any()
    close(got[~spoiled], o[~spoiled], tol[~spoiled])
    close(lse, e, et)
    again, _ = run(q, k, vv, starts)
    assert torch.equal(again.view(torch.int16), got.view(torch.int16)) and aqd.device_status() == 0


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dim,dtype", [(64, BF16), (128, F16), (192, BF16), (256, F16)])
def test_whole_rows_behind_a_query_and_queries_that_see_nothing(dim, dtype, layout):
    """More keys than queries, the diagonal anywhere in a tile; fewer keys than queries; the last keys and values NaN throughout."""
    lens, klens, last = [100, 300, 5, 200, 64], [377, 300, 131, 150, 3], [20, 100, 2, 149, 3]
    at, starts = starts_of(lens)
    kat, kstarts = starts_of(klens)
    q, k, v = inputs(dim, at[-1], kat[-1], 4, 2, dim, dtype)
    q = laid_out(q, layout)
    o, tol, e, et = reference(q, k, v, at, kat, True, 0.2)
    kk, vv = k.clone(), v.clone()
    clean = torch.zeros(at[-1], dtype=torch.bool, device="cuda")
    for i, n in enumerate(last):
        kk[kat[i + 1] - n:kat[i + 1]], vv[kat[i + 1] - n:kat[i + 1]] = math.nan, math.nan
        clean[at[i]:max(at[i], at[i + 1] - n)] = True
    got, lse = run(q, kk, vv, starts, kv_starts=kstarts, scale=0.2)
    close(got[clean], o[clean], tol[clean])
    close(lse[clean], e[clean], et[clean])
    assert got[~clean].isnan().all() and lse[~clean].isnan().all()
    assert (got[at[4]:at[5] - 3] == 0).all() and (lse[at[4]:at[5] - 3] == -math.inf).all()
    # without an order every query sees them
    got, _ = run(q, kk, vv, starts, kv_starts=kstarts, scale=0.2, causal=False)
    assert got.isnan().all()


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("every", [1, 3])
@pytest.mark.parametrize("dim,dtype", [(64, F16), (128, BF16), (192, BF16), (256, F16)])
def test_many_sequences_with_hidden_values(dim, dtype, every, layout):
    """More such jobs than a block keeps."""
    lens = [1 + i % 4 for i in range(1500)]
    at, starts = starts_of(lens)
    q, k, v = inputs(dim, at[-1], at[-1], 6, 2, dim, dtype)
    q = laid_out(q, layout)
    o, tol, e, et = reference(q, k, v, at, at, True, 0.1)
    vv, spoiled = v.clone(), torch.zeros(at[-1], dtype=torch.bool, device="cuda")
    ends = torch.tensor(at[1:], device="cuda")[::every] - 1
    vv[ends] = math.nan
    spoiled[ends] = True
    got, lse = run(q, k, vv, starts, scale=0.1)
    assert got[spoiled].isnan().all()
    close(got[~spoiled], o[~spoiled], tol[~spoiled])
    close(lse, e, et)
    assert aqd.device_status() == 0


@pytest.mark.parametrize("dim,dtype", [(64, BF16), (128, F16), (256, BF16)])
def test_nothing_but_nan(dim, dtype):
    """Values that are all NaN, and a long prompt whose last ones are."""
    at, starts = starts_of([3000, 40])
    q, k, v = inputs(dim, at[-1], at[-1], 4, 2, dim, dtype)
    o, tol, _, _ = reference(q, k, v, at, at, True, dim ** -0.5, set(range(2800, 2990)))
    got, _ = run(q, k, torch.full_like(v, math.nan), starts)
    assert got.isnan().all()
    vv = v.clone()
    vv[2990:3000] = math.nan
    got, _ = run(q, k, vv, starts)
    close(got[2800:2990], o[2800:2990], tol[2800:2990])
    assert got[2990:3000].isnan().all() and got[:2990].isfinite().all() and got[3000:].isfinite().all()
