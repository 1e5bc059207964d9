"""aqd_linear_int8 against the integer product: the sums are exact, and the scaled outputs are the stated float32
operations on them, so everything is compared bit for bit. (The reference product runs in float64, where sums below
2^53 are exact.)"""
import pytest
import torch

from paper_2007_06919_gb300 import aqd

pytestmark = pytest.mark.gpu


def codes(seed, rows, cols, kind="any"):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if kind == "any":
        return torch.randint(-128, 128, (rows, cols), generator=g, device="cuda").to(torch.int8)
    if kind == "quantized":
        return (32 * torch.randn(rows, cols, generator=g, device="cuda")).round().clamp(-127, 127).to(torch.int8)
    return torch.full((rows, cols), int(kind), dtype=torch.int8, device="cuda")


def scales(seed, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return 0.01 + torch.rand(n, generator=g, device="cuda")


def sums(x, w):
    return (x.double() @ w.double().T).to(torch.int64)


def scaled(s, xs, ws, bias, dtype):
    y = s.float() * xs[:, None] * ws
    if bias is not None:
        y = y + bias
    return y.to(dtype)


def check(x, w, layer=None, ws=True, dtypes=(torch.int32, torch.float32), bias=None):
    m, n = x.shape[0], w.shape[0]
    wsc, xs = scales(1, n), scales(2, m)
    layer = aqd.LinearWeights(w, wsc)
    space = aqd.linear_workspace(m, layer) if ws else None
    s = sums(x, w)
    for dt in dtypes:
        want = s.to(torch.int32) if dt == torch.int32 else scaled(s, xs, wsc, bias, dt)
        for _ in range(2):  # the second call finds what the first left in the workspace
            got = aqd.linear_int8(x, xs, layer, bias=bias, out_dtype=dt, workspace=space)
            torch.cuda.synchronize()
            assert aqd.device_status() == 0
            bad = (got != want).nonzero()
            assert not len(bad), f"{dt}: {len(bad)} of {got.numel()} differ, first at {bad[0].tolist()}"


M = [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 24, 31, 33, 64, 100, 127, 128, 129, 200, 255, 256, 257, 300, 511, 513, 1000]


@pytest.mark.parametrize("workspace", [True, False])
@pytest.mark.parametrize("m", M)
def test_tokens(m, workspace):
    check(codes(m, m, 1024), codes(m + 1, 640, 1024), ws=workspace)


@pytest.mark.parametrize("m", [1, 6, 20, 130, 700])
@pytest.mark.parametrize("n,k", [(1, 1), (1, 16), (3, 5), (16, 15), (17, 33), (100, 127), (127, 128), (129, 129), (255, 1000),
                                 (257, 2047), (1000, 2050), (2048, 64), (300, 4099), (33, 16384)])
def test_odd_sizes(m, n, k):
    check(codes(n, m, k), codes(k, n, k))
    check(codes(n, m, k), codes(k, n, k), ws=False, dtypes=(torch.int32,))


@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (16, 12288, 4096), (48, 4096, 12288), (513, 4096, 4096), (2048, 5120, 2048),
                                   (4096, 1024, 1024), (3000, 4100, 700)])
def test_layers(m, n, k):
    check(codes(m, m, k, "quantized"), codes(n, n, k, "quantized"), dtypes=(torch.int32, torch.bfloat16, torch.float16))


@pytest.mark.parametrize("m", [2, 16, 64, 300, 1024])
@pytest.mark.parametrize("k", [1024, 1040, 4096, 9000, 131071])
def test_largest_sums(k, m):
    """Every product at its largest magnitude, either sign: sums to the edge of int32."""
    n = 130
    lo, hi = codes(0, m, k, "-128"), codes(0, m, k, "127")
    w = torch.cat([codes(0, n // 2, k, "-128"), codes(0, n - n // 2, k, "127")])
    check(lo, w, dtypes=(torch.int32,))
    check(hi, w, dtypes=(torch.int32,))


@pytest.mark.parametrize("m", [4, 40, 400])
def test_sums_near_the_float32_limit(m):
    """Sums of odd values around 2^24, where a float32 running sum would drop their last bit."""
    k = 5000
    x, w = codes(1, m, k, "127"), codes(2, 200, k, "127")
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    w[:, 1040:] = torch.randint(-3, 4, (200, k - 1040), generator=g, device="cuda").to(torch.int8)
    check(x, w, dtypes=(torch.int32,))


@pytest.mark.parametrize("m", [1, 3, 8, 12, 70, 300])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_bias_and_types(m, dtype):
    check(codes(1, m, 320, "quantized"), codes(2, 200, 320, "quantized"), dtypes=(dtype,), bias=100 * (scales(3, 200) - 0.5))


@pytest.mark.parametrize("m", [1, 5, 40, 300])
@pytest.mark.parametrize("start,pad", [(0, 16), (0, 1), (1, 15), (3, 4), (16, 0)])
def test_strides_and_addresses(m, start, pad):
    k, n = 512, 200
    wide = codes(1, m, start + k + pad)
    x = wide[:, start:start + k]
    wcodes = codes(2, n, k + 3)[:, 3:]
    layer, xs = aqd.LinearWeights(wcodes, scales(1, n)), scales(2, m)
    want = scaled(sums(x, wcodes), xs, layer.scales, None, torch.bfloat16)
    for space in (None, aqd.linear_workspace(m, layer)):
        out = torch.full((m, n + 2 * 3), 7.0, dtype=torch.bfloat16, device="cuda")
        got = aqd.linear_int8(x, xs, layer, out=out[:, 3:3 + n], workspace=space)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert (out[:, :3] == 7).all() and (out[:, 3 + n:] == 7).all()


def test_leading_dimensions_and_broadcast_rows():
    w = codes(1, 70, 256)
    layer = aqd.LinearWeights(w, scales(1, 70))
    x = codes(2, 30, 256).view(2, 3, 5, 256)
    got = aqd.linear_int8(x, None, layer, out_dtype=torch.int32)
    assert got.shape == (2, 3, 5, 70)
    assert torch.equal(got.view(30, 70), sums(x.view(30, 256), w).int())
    one = codes(3, 1, 256).expand(40, 256)
    for space in (None, aqd.linear_workspace(40, layer)):
        assert torch.equal(aqd.linear_int8(one, None, layer, out_dtype=torch.int32, workspace=space), sums(one, w).int())


def test_scales_pass_through():
    """NaN and infinite scales reach their rows and columns and no others; scales may change between calls."""
    x, w = codes(1, 20, 128, "quantized"), codes(2, 90, 128, "quantized")
    xs, wsc = scales(1, 20), scales(2, 90)
    layer = aqd.LinearWeights(w, wsc)
    xs[3] = float("nan")
    wsc[7] = float("inf")
    got = aqd.linear_int8(x, xs, layer, out_dtype=torch.float32)
    want = scaled(sums(x, w), xs, wsc, None, torch.float32)
    torch.cuda.synchronize()
    assert torch.equal(got.nan_to_num(-1e30, 1e30, -2e30), want.nan_to_num(-1e30, 1e30, -2e30))


def test_a_workspace_serves_other_sizes():
    w = codes(1, 500, 2048)
    layer = aqd.LinearWeights(w, scales(1, 500))
    space = aqd.linear_workspace(900, layer)
    for m in (900, 1, 30, 513, 64, 900):
        x = codes(m, m, 2048)
        got = aqd.linear_int8(x, None, layer, out_dtype=torch.int32, workspace=space)
        torch.cuda.synchronize()
        assert torch.equal(got, sums(x, w).int()), m


def test_offsets_past_32_bits():
    m, k, n = 3, 256, 64
    buf = torch.empty((m - 1) * 2_500_000_000 + k, dtype=torch.int8, device="cuda")
    w = codes(1, n, k)
    layer = aqd.LinearWeights(w, scales(1, n))
    x = buf.as_strided((m, k), (2_500_000_000, 1))
    x.copy_(codes(2, m, k))
    want = sums(x.contiguous(), w).int()
    assert torch.equal(aqd.linear_int8(x, None, layer, out_dtype=torch.int32), want)
    out = torch.empty((m - 1) * 1_200_000_000 + n, dtype=torch.int32, device="cuda").as_strided((m, n), (1_200_000_000, 1))
    xc = x.contiguous()
    assert torch.equal(aqd.linear_int8(xc, None, layer, out=out), want)


def test_from_float_and_no_tokens():
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    w = torch.randn(96, 320, generator=g, device="cuda")
    layer = aqd.LinearWeights.from_float(w)
    eye = torch.eye(320, device="cuda").mul(127).to(torch.int8)
    got = aqd.linear_int8(eye, torch.full((320,), 1 / 127, device="cuda"), layer, out_dtype=torch.float32)
    # half a step of each channel, and float32's own roundings of values up to 127 steps
    assert ((got.T - w).abs() <= (0.5 + 1e-3) * layer.scales[:, None]).all()
    empty = aqd.linear_int8(torch.empty(0, 320, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"), layer)
    assert empty.shape == (0, 96)


def test_streams_and_graphs():
    x, w = codes(1, 40, 2048), codes(2, 384, 2048)
    layer = aqd.LinearWeights(w, scales(1, 384))
    space = aqd.linear_workspace(40, layer)
    want = sums(x, w).int()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = aqd.linear_int8(x, None, layer, out_dtype=torch.int32, workspace=space, stream=s)
    s.synchronize()
    assert torch.equal(got, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = aqd.linear_int8(x, None, layer, out_dtype=torch.int32, workspace=space)
    for _ in range(3):
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
    assert aqd.device_status() == 0


def test_refusals():
    w = codes(1, 64, 128)
    layer = aqd.LinearWeights(w, scales(1, 64))
    x, xs = codes(2, 4, 128), scales(2, 4)
    bad = [lambda: aqd.linear_int8(x.float(), xs, layer), lambda: aqd.linear_int8(x[:, :64], xs, layer),
           lambda: aqd.linear_int8(x, xs[:2], layer), lambda: aqd.linear_int8(x, None, layer),
           lambda: aqd.linear_int8(x, xs.double(), layer), lambda: aqd.linear_int8(x, xs, layer, bias=xs),
           lambda: aqd.linear_int8(x, xs, layer, out=torch.empty(4, 63, device="cuda")),
           lambda: aqd.linear_int8(x, xs, layer, out_dtype=torch.float64), lambda: aqd.linear_int8(x.cpu(), xs, layer),
           lambda: aqd.linear_int8(x.t(), xs, layer), lambda: aqd.LinearWeights(w.float(), scales(1, 64)),
           lambda: aqd.LinearWeights(w, scales(1, 63)), lambda: aqd.LinearWeights(w[0], scales(1, 64))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    out = torch.empty(64, device="cuda").expand(4, 64)
    with pytest.raises(aqd.AqdError):
        aqd.linear_int8(x, xs, layer, out=out)
