"""The norm with eps = 0 of rows whose squares lie below float32's range: their normalized values are ordinary ones. Compared as the other rows
are, with the formula in 64 bits."""
import pytest
import torch

from paper_2007_06919_gb300 import aqd
from test_gpu_lm_rows import check, norm64, normal

pytestmark = pytest.mark.gpu

# a row's size; its largest value times its weight is above 2^-120 = 7.5e-37, below which a row has no codes
SIZES = [1.0, 1e-12, 3e-18, 1e-19, 3e-20, 1e-20, 1e-21, 1e-23, 1e-27, 1e-30, 1e-34, 3e-36, 1e4]
# a warp's rows, a block's, in shared memory, in a cluster's, read twice
COLS = [64, 1000, 4096, 8192, 12288, 20000, 40000, 150000, 400000]


def rows(seed, cols, dtype):
    return (normal(seed, len(SIZES), cols).double() * torch.tensor(SIZES, dtype=torch.float64, device="cuda")[:, None]).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", COLS)
def test_whole_rows(cols, dtype):
    x, r, w = rows(1, cols, dtype), rows(2, cols, dtype), (1 + 0.3 * normal(3, cols)).to(dtype)
    q = aqd.rms_norm_quant(x, w, eps=0.0, values=torch.float32)
    check(q, norm64(x.double(), w, 0.0), torch.float32)
    q = aqd.rms_norm_quant(x, w, eps=0.0, residual=r)
    check(q, norm64(x.double() + r.double() if dtype != torch.float32 else (x + r).double(), w, 0.0), None)
    assert q.values is None
    again = aqd.rms_norm_quant(x, w, eps=0.0, residual=r, summed=x)
    torch.cuda.synchronize()
    assert torch.equal(again.codes, q.codes) and torch.equal(again.scales, q.scales) and torch.equal(x, q.summed)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [5, 301, 1003, 9001, 18001, 70001])
def test_rows_that_lie_otherwise(cols, dtype):
    """Odd widths; the halves of odd rows; a sum that lies otherwise than the codes."""
    x, r, w = rows(1, cols, dtype), rows(2, cols, dtype), (1 + 0.3 * normal(3, cols)).to(dtype)
    h = norm64(x.double() + r.double() if dtype != torch.float32 else (x + r).double(), w, 0.0)
    s = torch.empty(len(SIZES), cols + 3, dtype=dtype, device="cuda")[:, 1:1 + cols]
    a, b = torch.cat([x, r], 1).chunk(2, dim=1)
    for q in (aqd.rms_norm_quant(x, w, eps=0.0, residual=r), aqd.rms_norm_quant(a, w, eps=0.0, residual=b),
              aqd.rms_norm_quant(x, w, eps=0.0, residual=r, summed=s)):
        check(q, h, None)


@pytest.mark.parametrize("cols", [64, 1003, 8192, 40000, 400000])
def test_one_value_and_small_eps(cols):
    """A single value in a row of zeros; eps that float32 can just hold, and one that counts beside the squares."""
    w = torch.ones(cols, device="cuda")
    x = torch.zeros(4, cols, device="cuda")
    x[0, cols // 2], x[1, 0], x[2, cols - 1] = 1e-30, -1e-22, 3e-36
    q = aqd.rms_norm_quant(x, w, eps=0.0)
    torch.cuda.synchronize()
    check(aqd.RowCodes(q.codes[:3], q.scales[:3]), norm64(x[:3].double(), w, 0.0), None)
    assert q.scales[3] == 0 and (q.codes[3] == 0).all()
    y = rows(4, cols, torch.float32)
    for eps in (1e-45, 1e-40, 2e-38, 1e-36, 1e-30):
        eps = torch.tensor(eps).item()  # as float32 has it
        check(aqd.rms_norm_quant(y, w, eps=eps), norm64(y.double(), w, eps), None)
