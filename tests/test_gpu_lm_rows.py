"""The row quantizers (aqd_quant_rows, aqd_rms_norm_quant, aqd_gated_act_quant) against their formulas in 64 bits.

What is compared, and how near:
  * a code is u * 127 / a rounded to nearest. u and a carry a few float32 roundings (the activation's exponential or hyperbolic
    tangent among them: at most 16 units of 2^-24 of |gate * up|, itself at most 8 a in these rows), so a code lies within 1/2 + 127 * 16 * 8 * 2^-24
    < 1/2 + 1e-3 of the exact quotient;
  * the scale: a sum of squares in float32 adds at most (terms per thread + 16) roundings, under a square root half of that, and 16
    more elsewhere: within (cols / 64 + 32) * 2^-24 of its size;
  * values are code * scale in float32 rounded to their type, and the sum x + residual likewise: bit for bit."""
import math

import pytest
import torch

from paper_2007_06919_gb300 import aqd

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
# one element, one vector and its neighbours, whole and partial blocks, past what a block keeps in registers
COLS = [1, 2, 7, 8, 9, 64, 100, 257, 1000, 1024, 1025, 2048, 4096, 4097, 5120, 8192, 12288, 16384, 16387, 32768, 40008, 70001]


def normal(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def check(q, u, vtype):
    """q against the rows u (float64), all of them finite and large enough to have codes."""
    torch.cuda.synchronize()
    cols = u.shape[-1]
    a = u.abs().amax(-1, keepdim=True)
    assert q.codes.dtype == torch.int8 and q.codes.shape == u.shape and q.scales.shape == u.shape[:-1]
    off = (q.codes.double() - torch.where(a > 0, u * 127 / a, 0.0)).abs().max().item()
    assert off <= 0.5 + 1e-3
    want = a.squeeze(-1) / 127
    assert ((q.scales.double() - want).abs() <= (cols / 64 + 32) * 2.0 ** -24 * want).all()
    if q.values is not None:
        assert q.values.dtype == vtype
        assert torch.equal(q.values, (q.codes.float() * q.scales.unsqueeze(-1)).to(vtype))


def norm64(h, w, eps):
    return h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps) * w.double()


def act64(g, act):
    if act == "silu":
        return g / (1 + torch.exp(-g))
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_norm(cols, dtype):
    for rows in (1, 3):
        x, r = (3 * normal(cols, rows, cols)).to(dtype), normal(cols + 1, rows, cols).to(dtype)
        w = (1 + 0.3 * normal(cols + 2, cols)).to(dtype)
        q = aqd.rms_norm_quant(x, w, eps=1e-5, residual=r, values=True)
        check(q, norm64(x.double() + r.double() if dtype != torch.float32 else (x + r).double(), w, 1e-5), dtype)
        assert torch.equal(q.summed, (x.float() + r.float()).to(dtype))
        q = aqd.rms_norm_quant(x, w, eps=0.0)
        check(q, norm64(x.double(), w, 0.0), dtype)
        assert q.values is None and q.summed is None


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_gated(cols, dtype, act):
    both = (2 * normal(cols, 3, 2 * cols)).to(dtype)
    # every row's largest value is well away from zero
    both[:, 0] = 3.0
    both[:, cols] = 4.0
    gate, up = both.chunk(2, dim=1)
    q = aqd.gated_act_quant(gate, up, act=act, values=torch.float32)
    check(q, act64(gate.double(), act) * up.double(), torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_plain(cols, dtype):
    x = normal(cols, 5, cols).to(dtype)
    q = aqd.quant_rows(x, values=torch.bfloat16)
    check(q, x.double(), torch.bfloat16)
    v = aqd.quant_rows(x, codes=False, values=torch.bfloat16)
    torch.cuda.synchronize()
    assert v.codes is None and torch.equal(v.values, q.values) and torch.equal(v.scales, q.scales)


@pytest.mark.parametrize("rows", [1, 2, 151, 152, 153, 1217, 5000])
@pytest.mark.parametrize("cols", [48, 520, 3000])
def test_many_rows(rows, cols):
    x, r = normal(1, rows, cols).bfloat16(), normal(2, rows, cols).bfloat16()
    w = normal(3, cols)  # float32 weights beside bfloat16 rows
    q = aqd.rms_norm_quant(x, w, residual=r, values=torch.float16)
    check(q, norm64(x.double() + r.double(), w, 1e-6), torch.float16)


@pytest.mark.parametrize("cols", [96, 1003, 4096, 20000])
@pytest.mark.parametrize("start", [0, 1, 8])
@pytest.mark.parametrize("pad", [0, 1, 8, 24])
def test_strides_and_addresses(cols, start, pad):
    """Rows of a wider matrix, at whole and odd addresses, every output with a stride of its own; nothing else is written."""
    rows, dtype = 9, torch.bfloat16

    def view(fill, dt, p):
        m = torch.full((rows, start + cols + p), fill, dtype=dt, device="cuda")
        return m, m[:, start:start + cols]
    (_, x), (_, r) = view(0, dtype, pad), view(0, dtype, pad + 8)
    x.copy_(normal(4, rows, cols))
    r.copy_(normal(5, rows, cols))
    w = torch.empty(cols + 1, dtype=dtype, device="cuda")[1:]
    w.copy_(1 + 0.1 * normal(6, cols))
    whole, s = view(7.0, dtype, pad)
    q = aqd.rms_norm_quant(x, w, residual=r, summed=s, values=True)
    check(q, norm64(x.double() + r.double(), w, 1e-6), dtype)
    assert torch.equal(s, (x.float() + r.float()).to(dtype))
    assert (whole[:, :start] == 7).all() and (whole[:, start + cols:] == 7).all()
    g = aqd.gated_act_quant(x, r)
    check(g, act64(x.double(), "silu") * r.double(), None)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(700, 257), (700, 515), (310, 1537), (9, 1539), (400, 5003), (330, 8189), (5, 8189), (320, 9215), (3, 9213), (310, 18425)])
def test_rows_that_start_inside_a_vector(rows, cols, dtype):
    """Adjacent rows of odd widths: every tensor's rows start at the same place in their vectors, which is another for every row."""
    x, r = normal(11, rows, cols).to(dtype), normal(12, rows, cols).to(dtype)
    w = (1 + 0.3 * normal(13, cols)).to(dtype)
    h = x.double() + r.double() if dtype != torch.float32 else (x + r).double()
    q = aqd.rms_norm_quant(x, w, residual=r, values=True)
    check(q, norm64(h, w, 1e-6), dtype)
    assert torch.equal(q.summed, (x.float() + r.float()).to(dtype))
    check(aqd.rms_norm_quant(x, w, values=torch.float32), norm64(x.double(), w, 1e-6), torch.float32)
    check(aqd.quant_rows(x, values=torch.bfloat16), x.double(), torch.bfloat16)
    x[:, 0], r[:, 0] = 3.0, 4.0
    check(aqd.gated_act_quant(x, r, act="gelu_tanh", values=True), act64(x.double(), "gelu_tanh") * r.double(), dtype)
    # whole vectors around the matrix stay as they are
    room = torch.full((rows * cols + 64,), 7.0, dtype=dtype, device="cuda")
    s = room[32:32 + rows * cols].view(rows, cols)
    aqd.rms_norm_quant(x, w, residual=r, summed=s)
    torch.cuda.synchronize()
    assert torch.equal(s, (x.float() + r.float()).to(dtype)) and (room[:32] == 7).all() and (room[32 + rows * cols:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [2049, 3335, 6001, 9001])
def test_inputs_that_lie_otherwise_than_the_outputs(cols, dtype):
    """The two halves of rows of an odd width, and of a wider matrix: the inputs start at other places in their vectors than the outputs."""
    rows = 37
    both = normal(14, rows, 2 * cols).to(dtype)
    x, r = both.chunk(2, dim=1)
    w = (1 + 0.3 * normal(15, cols)).to(dtype)
    h = x.double() + r.double() if dtype != torch.float32 else (x + r).double()
    q = aqd.rms_norm_quant(x, w, residual=r, values=True)
    check(q, norm64(h, w, 1e-6), dtype)
    assert torch.equal(q.summed, (x.float() + r.float()).to(dtype))
    check(aqd.quant_rows(r, values=torch.float32), r.double(), torch.float32)
    v = aqd.quant_rows(r, codes=False, values=torch.float16)
    torch.cuda.synchronize()
    assert torch.equal(v.values, aqd.quant_rows(r, values=torch.float16).values)
    wide = normal(16, rows, cols + 5).to(dtype)[:, 3:3 + cols]
    wide[:, 0], x[:, 0] = 3.0, 4.0
    check(aqd.gated_act_quant(wide, x, values=True), act64(wide.double(), "silu") * x.double(), dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 18440), (310, 24576), (7, 36872), (2, 73736), (320, 40960), (3, 147440), (1, 300000)])
def test_rows_of_several_blocks(rows, cols, dtype):
    x, r = normal(17, rows, cols).to(dtype), normal(18, rows, cols).to(dtype)
    w = (1 + 0.3 * normal(19, cols)).to(dtype)
    x[0, cols - 1] = 9.0  # the largest is in the last block's part
    h = x.double() + r.double() if dtype != torch.float32 else (x + r).double()
    q = aqd.rms_norm_quant(x, w, residual=r, values=True)
    check(q, norm64(h, w, 1e-6), dtype)
    assert torch.equal(q.summed, (x.float() + r.float()).to(dtype))
    check(aqd.rms_norm_quant(x, w), norm64(x.double(), w, 1e-6), None)
    check(aqd.quant_rows(x, values=torch.float32), x.double(), torch.float32)
    again = aqd.rms_norm_quant(x, w, residual=r, values=True, summed=x)
    torch.cuda.synchronize()
    assert torch.equal(again.codes, q.codes) and torch.equal(again.scales, q.scales) and torch.equal(x, q.summed)
    x[:, 0], r[:, 0] = 3.0, 4.0
    check(aqd.gated_act_quant(x, r, values=True), act64(x.double(), "silu") * r.double(), dtype)
    x[rows - 1, cols // 2] = math.nan
    q = aqd.quant_rows(x)
    torch.cuda.synchronize()
    assert q.scales[rows - 1].isnan() and (q.codes[rows - 1] == 0).all() and q.scales[:rows - 1].isfinite().all()


def test_more_long_rows_than_a_grid_has():
    one = normal(20, 1, 40000).half()
    q = aqd.quant_rows(one.expand(65539, 40000))
    torch.cuda.synchronize()
    check(aqd.RowCodes(q.codes[:1], q.scales[:1]), one.double(), None)
    assert (q.scales == q.scales[0]).all()
    for at in (0, 65534, 65535, 65538):
        assert torch.equal(q.codes[at], q.codes[0])


def test_leading_dimensions_and_broadcast_rows():
    x, w = normal(7, 2, 5, 3, 96).half(), torch.ones(96, device="cuda")
    check(aqd.rms_norm_quant(x, w), norm64(x.double(), w, 1e-6), None)
    one = normal(8, 1, 640).expand(6, 640)  # one row's memory read as six
    check(aqd.quant_rows(one), one.double(), None)
    check(aqd.quant_rows(x[:, :, 1]), x[:, :, 1].double(), None)
    v = normal(9, 333)
    check(aqd.quant_rows(v), v.double(), None)


@pytest.mark.parametrize("which", ["x", "residual"])
@pytest.mark.parametrize("cols", [64, 1001, 4096, 50000])
def test_sum_in_place(cols, which):
    x, r = normal(1, 33, cols).bfloat16(), normal(2, 33, cols).bfloat16()
    w = (1 + 0.1 * normal(3, cols)).bfloat16()
    want = aqd.rms_norm_quant(x, w, residual=r)
    x2, r2 = x.clone(), r.clone()
    q = aqd.rms_norm_quant(x2, w, residual=r2, summed=x2 if which == "x" else r2)
    torch.cuda.synchronize()
    assert torch.equal(q.summed, want.summed) and torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales)
    assert torch.equal(r2 if which == "x" else x2, r if which == "x" else x)


@pytest.mark.parametrize("cols", [5, 512, 1003, 4096, 40000])
def test_rows_of_zeros_tiny_values_and_non_finite_values(cols):
    x = normal(1, 8, cols)
    x[0] = 0
    x[1] = 2.0 ** -130
    x[2, cols // 2] = math.nan
    x[3, cols - 1] = math.inf
    x[4, 0] = -math.inf
    x[5] = 0
    x[5, cols - 1] = 2.0 ** -119
    w = torch.ones(cols, device="cuda")
    for q in (aqd.quant_rows(x, values=True), aqd.rms_norm_quant(x, w, values=True),
              aqd.gated_act_quant(torch.full_like(x, 40.0), x / 40, values=True)):
        torch.cuda.synchronize()
        assert (q.codes[:5] == 0).all() and (q.scales[:2] == 0).all() and (q.values[:2] == 0).all()
        assert q.scales[2:5].isnan().all() and q.values[2:5].isnan().all()
        assert q.scales[6:].isfinite().all() and (q.codes[6:].abs().amax(1) == 127).all()
    q = aqd.quant_rows(x)
    torch.cuda.synchronize()
    assert q.codes[5, -1] == 127 and q.codes[5].abs().sum() == 127 and q.scales[5].item() > 0


def test_large_values():
    """Products beyond the inputs' range stay finite in float32."""
    x = (60000 * torch.sign(normal(1, 4, 4096))).half()
    q = aqd.gated_act_quant(x.abs(), x)
    check(q, x.double().abs() * x.double(), None)
    b = torch.full((2, 1024), 1e30, device="cuda")
    q = aqd.rms_norm_quant(b, torch.ones(1024, device="cuda"))  # the squares pass float32
    torch.cuda.synchronize()
    assert q.scales.isnan().all() and (q.codes == 0).all()


def test_offsets_past_32_bits():
    """Rows whose elements lie beyond 2^32 bytes and 2^31 elements from the first."""
    rows, cols, ld = 4, 1000, 900_000_001
    buf = torch.empty((rows - 1) * ld + cols, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((rows, cols), (ld, 1))
    x.copy_(normal(3, rows, cols))
    check(aqd.quant_rows(x), x.double(), None)
    w = torch.ones(cols, device="cuda")
    check(aqd.rms_norm_quant(x, w, residual=x), norm64(2 * x.double(), w, 1e-6), None)
    check(aqd.gated_act_quant(x, x), act64(x.double(), "silu") * x.double(), None)


def test_no_rows():
    x, w = torch.empty(0, 64, device="cuda"), torch.ones(64, device="cuda")
    for q in (aqd.quant_rows(x), aqd.rms_norm_quant(x, w, residual=x), aqd.gated_act_quant(x, x)):
        assert q.codes.shape == (0, 64) and q.scales.shape == (0,)


def test_other_streams_and_graphs():
    x, w = normal(1, 64, 4096).bfloat16(), torch.ones(4096, device="cuda")
    want = aqd.rms_norm_quant(x, w)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = aqd.rms_norm_quant(x, w, stream=s)
    s.synchronize()
    assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        q = aqd.rms_norm_quant(x, w)
    x.mul_(-1)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(q.codes, -want.codes)


def test_refusals():
    x, w = normal(1, 4, 64), torch.ones(64, device="cuda")
    bad = [lambda: aqd.quant_rows(x.double()), lambda: aqd.quant_rows(x.t()), lambda: aqd.quant_rows(x.cpu()),
           lambda: aqd.quant_rows(x, values=torch.int8), lambda: aqd.quant_rows(x, codes=False),
           lambda: aqd.rms_norm_quant(x, w[:32]), lambda: aqd.rms_norm_quant(x, w, residual=x.half()),
           lambda: aqd.rms_norm_quant(x, w, residual=x[:2]), lambda: aqd.rms_norm_quant(x, w.int()),
           lambda: aqd.rms_norm_quant(x, w, residual=x, summed=x.half()), lambda: aqd.gated_act_quant(x, x, act="relu"),
           lambda: aqd.gated_act_quant(x, x[:, :32]), lambda: aqd.quant_rows(x[:, :0]),
           lambda: aqd.quant_rows(normal(1, 3, 4, 64)[:, :2]), lambda: aqd.quant_rows(torch.tensor(1.0, device="cuda"))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(aqd.AqdError):
        aqd.rms_norm_quant(x, w, eps=-1.0)
    with pytest.raises(aqd.AqdError):  # rows of the sum that overlap
        aqd.rms_norm_quant(x, w, residual=x, summed=torch.empty(64, device="cuda").expand(4, 64))
