"""Norms and rotation of heads, and the 4-bit cache's rows, against the formulas in 64 bits."""
import math

import pytest
import torch

from attention_ref import U, close, held, rotated
from paper_2007_06919_gb300 import aqd

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


def freqs(rot):
    return (10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / max(rot, 1))).float()


def inputs(seed, tokens, heads, kv, dim, dtype, pad=0):
    """Views of one product's rows, whose rows start `pad` elements into it."""
    torch.manual_seed(seed)
    both = (2 * torch.randn(tokens, (heads + 2 * kv) * dim + pad, device="cuda")).to(dtype)[:, pad:]
    both = both.unflatten(1, (heads + 2 * kv, dim))
    return both[:, :heads], both[:, heads:heads + kv], both[:, heads + kv:]


# A result's two parts carry: the sum of squares (a tree, below 12 roundings), division, root (2 steps), two products, sine and cosine (2 steps of 2^-24 and an
# angle off by 2 pi 2^-25), the product and the sum: below 32 half steps of float32 of the parts' size; then one rounding to the type, whose half step
# is relative down to the type's least normal value: float16's values below 2^-14 are 2^-24 apart, so a rounding there moves one by up to 2^-25.
def bound(want, size, dtype):
    return U[dtype] * want.abs() + 32 * 2.0 ** -24 * size + (2.0 ** -25 if dtype is F16 else 1e-30)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,kv,dim,rot,dtype,pad", [
    (1, 32, 8, 128, 128, BF16, 0), (5, 7, 1, 64, 64, F16, 0), (700, 4, 2, 128, 32, BF16, 0), (33, 3, 3, 256, 256, F32, 0),
    (9, 14, 2, 80, 40, BF16, 0), (3, 2, 1, 2, 2, F32, 0), (17, 5, 5, 6, 4, F16, 0), (21, 8, 4, 128, 128, BF16, 1),
    (13, 2, 2, 512, 512, F32, 0), (13, 2, 2, 512, 96, F16, 0), (50, 6, 2, 130, 130, BF16, 0), (19, 4, 4, 192, 48, F16, 0),
    (40, 9, 3, 64, 0, BF16, 0), (2000, 2, 1, 64, 62, F16, 0), (11, 1, 1, 96, 10, F32, 3)])
def test_norm_and_rotation(tokens, heads, kv, dim, rot, dtype, pad, interleaved):
    q, k, _ = inputs(tokens + dim, tokens, heads, kv, dim, dtype, pad)
    wq, wk = ((1 + 0.3 * torch.randn(dim, device="cuda")).to(dtype) for _ in range(2))
    pos = torch.randint(0, 1 << 20, (tokens,), device="cuda")
    f = freqs(rot) if rot else None
    for weights in ((wq, wk), (None, None), (wq, None)):
        out = aqd.qk_norm_rope(q, k, pos if rot else None, f, q_weight=weights[0], k_weight=weights[1], interleaved=interleaved)
        for x, w, got in ((q, weights[0], out.q), (k, weights[1], out.k)):
            want, size = rotated(x, w, pos, f, interleaved, 1e-6)
            close(got, want, bound(want, size, dtype))


def test_far_and_negative_positions():
    q, k, _ = inputs(0, 12, 2, 2, 64, F32)
    pos = torch.tensor([0, 1, -1, 2 ** 20, -(2 ** 20) + 3, 2 ** 27, 2 ** 27 + 1, 5, 2 ** 24 + 1, 2 ** 26 - 7, -5, 7], device="cuda")
    f = freqs(64)
    out = aqd.qk_norm_rope(q, k, pos, f)
    want, size = rotated(q, None, pos, f, False, 0)
    close(out.q, want, bound(want, size, F32))
    pos = pos * 1000  # beyond 2^37, slow frequencies alone
    f = freqs(64) * 1e-3
    out = aqd.qk_norm_rope(q, k, pos, f)
    want, size = rotated(q, None, pos, f, False, 0)
    close(out.q, want, bound(want, size, F32))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("pad", [0, 1])
def test_in_place_and_other_layouts(dtype, pad):
    q, k, v = inputs(3, 37, 6, 2, 128, dtype, pad)
    w = (1 + 0.3 * torch.randn(128, device="cuda")).float()
    pos, f = torch.arange(37, device="cuda"), freqs(128)
    want = aqd.qk_norm_rope(q, k, pos, f, q_weight=w, k_weight=w)
    turned = q.transpose(0, 1).contiguous().transpose(0, 1)  # [heads][tokens]
    out = torch.full((6, 37, 130), 7.0, device="cuda", dtype=dtype)
    got = aqd.qk_norm_rope(turned, k, pos, f, q_weight=w, k_weight=w, q_out=out[..., :128].transpose(0, 1))
    # (rows that start elsewhere may sum their squares in another order: each within the bound of the formula)
    for a, b, x in ((got.q, want.q, q), (got.k, want.k, k)):
        exact, size = rotated(x, w, pos, f, False, 1e-6)
        close(a, exact, bound(exact, size, dtype))
        close(b, exact, bound(exact, size, dtype))
    assert (out[..., 128:] == 7).all()
    kept = v.clone()
    same = aqd.qk_norm_rope(q, k, pos, f, q_weight=w, k_weight=w, q_out=q, k_out=k)
    assert same.q.data_ptr() == q.data_ptr() and torch.equal(q, want.q) and torch.equal(k, want.k) and torch.equal(v, kept)


def test_norm_eps_and_special_rows():
    q, k, _ = inputs(4, 6, 2, 1, 64, BF16)
    q, k = q.clone(), k.clone()
    q[0] = 0
    q[1, 0, 3] = math.nan
    q[2, 1, 5] = math.inf
    q[3] *= 1e-20
    w = torch.ones(64, device="cuda", dtype=BF16)
    out = aqd.qk_norm_rope(q, k, None, None, q_weight=w, k_weight=w, eps=1e-6).q
    assert (out[0] == 0).all() and out[1, 0].isnan().all() and not out[1, 1].isnan().any() and out[2, 1, 5].isnan()
    want, size = rotated(q[3:], w, None, None, False, 1e-6)
    close(out[3:], want, bound(want, size, BF16))


# ------------------------------------------------------------------ the cache


def slots_for(cache, tokens, seed=0):
    torch.manual_seed(seed)
    return torch.randperm(cache.pages * cache.page_size, device="cuda")[:tokens]


def check_held(got, x):
    """Exactly the values of the definition; beside a tie the other code's too."""
    codes, low, step, tie = held(x)
    want = (low + step * codes).float().to(got.dtype)
    other = [(low + step * (codes + d)).float().to(got.dtype) for d in (-1, 1)]
    assert ((got == want) | (tie & ((got == other[0]) | (got == other[1])))).all()


# Spans a little over 15 times a bfloat16, which float32 rounds down to it: the step is the next one.
@pytest.mark.parametrize("dtype,low,high", [(F32, -8.0, 7 + 2.0 ** -21), (F32, -2.0 ** -30, 15.0), (F16, -2.0 ** -24, 15.0), (BF16, -2.0 ** -40, 30.0), (F32, -3.0, 12 + 2.0 ** -20),
                                            (F32, 0.0, 15 + 2.0 ** -20), (F32, -8.0, 7 - 2.0 ** -21)])
@pytest.mark.parametrize("pad", [0, 1])
def test_step_of_a_span_just_over_fifteen(dtype, low, high, pad):
    cache = aqd.KVCache(2, 16, 2, 64)
    _, k, v = inputs(5, 9, 1, 2, 64, dtype, pad)
    k, v = (x.abs().clamp(0.5, 6.5) for x in (k, v))
    k[..., 5], k[..., 60], v[..., 31], v[..., 0] = low, high, low, high
    slots = slots_for(cache, 9)
    aqd.cache_write(cache, k, v, slots)
    gk, gv = aqd.cache_read(cache, slots, dtype=F32)
    check_held(gk, k)
    check_held(gv, v)


@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("tokens,kv,dim,page,dtype", [(1, 8, 128, 64, BF16), (100, 2, 64, 16, F16), (77, 3, 192, 32, F32), (300, 1, 256, 1024, BF16),
                                                      (1000, 5, 128, 128, F32), (40, 4, 64, 256, BF16)])
def test_write_and_read(tokens, kv, dim, page, dtype, pad):
    cache = aqd.KVCache(-(-2 * tokens // page) + 1, page, kv, dim)
    cache.data.fill_(0xA5)
    _, k, v = inputs(tokens, tokens, 1, kv, dim, dtype, pad)
    slots = slots_for(cache, tokens)
    aqd.cache_write(cache, k, v, slots)
    for out in (F32, F16, BF16):
        gk, gv = aqd.cache_read(cache, slots, dtype=out)
        check_held(gk, k)
        check_held(gv, v)
    # the other places keep their bytes
    rest = torch.ones(cache.pages * page, dtype=torch.bool, device="cuda")
    rest[slots] = False
    ok, ov = aqd.cache_read(cache, rest.nonzero().flatten(), dtype=F32)
    assert torch.equal(ok, ok[:1, :1, :2].repeat(ok.shape[0], kv, dim // 2)) and torch.equal(ov, ok)


@pytest.mark.parametrize("pad,rot,interleaved", [(0, 128, False), (0, 128, True), (1, 128, False), (0, 20, False), (0, 6, True)])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_one_pass_writes_what_two_do(dtype, pad, rot, interleaved):
    q, k, v = inputs(8, 53, 4, 2, 128, dtype, pad)
    w = 1 + 0.3 * torch.randn(128, device="cuda")
    pos, f = torch.arange(53, device="cuda") + 1000, freqs(rot)
    one, two = (aqd.KVCache(5, 32, 2, 128) for _ in range(2))
    one.data.zero_(), two.data.zero_()
    slots = slots_for(one, 53)
    slots[7], slots[9], slots[11] = -1, one.pages * 32, 1 << 60  # skipped
    args = dict(q_weight=w, k_weight=w, interleaved=interleaved)
    want = aqd.qk_norm_rope(q, k, pos, f, **args)
    aqd.cache_write(two, want.k, v, slots)
    got = aqd.qk_norm_rope(q, k, pos, f, v=v, cache=one, slots=slots, **args)
    assert got.k is None and torch.equal(got.q, want.q) and torch.equal(one.data, two.data)
    both = aqd.qk_norm_rope(q, k, pos, f, v=v, cache=one, slots=slots, k_out=torch.empty_like(want.k), **args)
    assert torch.equal(both.k, want.k) and torch.equal(one.data, two.data)
    gone = aqd.cache_read(one, torch.tensor([-1, one.pages * 32, -(1 << 62)], device="cuda"))
    assert (gone[0] == 0).all() and (gone[1] == 0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_special_rows(dtype):
    rows = torch.randn(12, 1, 64, device="cuda")
    rows[0] = 0
    rows[1] = 3.0
    rows[2] = 1.0 / 3
    rows[3, 0, 5] = math.nan
    rows[4, 0, 5] = math.inf
    rows[5, 0, 5] = -math.inf
    rows[6] = rows[6] * 1e-30 + 5
    rows[7, 0, 0], rows[7, 0, 1] = 3e38, -3e38
    rows[8] *= 1e-38
    rows[9] *= 1e30
    rows[10] = -7.0
    rows[11, 0, :] = torch.arange(64, device="cuda") % 16 - 3.0  # every code, no rounding
    x = rows.to(dtype)
    cache = aqd.KVCache(1, 16, 1, 64)
    slots = torch.arange(12, device="cuda")
    aqd.cache_write(cache, x, x, slots)
    for got in aqd.cache_read(cache, slots, dtype=F32):
        for r in (3, 4, 5, 7):
            assert got[r].isnan().all()
        fine = torch.tensor([r for r in range(12) if r not in (3, 4, 5, 7)], device="cuda")
        check_held(got[fine], x[fine])
        assert torch.equal(got[11], rows[11]) and (got[0] == 0).all() and (got[1] == 3).all() and (got[10] == -7).all()
        _, _, step, _ = held(x[fine])
        assert ((got[fine].double() - x[fine].double()).abs() <= 0.5 * step + 2.0 ** -23 * x[fine].double().abs()).all()


def test_offsets_past_32_bits():
    cache = aqd.KVCache(70_000, 64, 8, 128)  # 4.9 GB
    assert cache.data.numel() > 1 << 32
    _, k, v = inputs(9, 6, 1, 8, 128, BF16)
    last = cache.pages * 64
    slots = torch.tensor([0, last - 1, last - 65, last // 2, (1 << 32) // 1088 + 1, 63], device="cuda")
    aqd.cache_write(cache, k, v, slots)
    gk, gv = aqd.cache_read(cache, slots)
    check_held(gk, k)
    check_held(gv, v)


def test_no_tokens():
    cache = aqd.KVCache(1, 16, 2, 64)
    e = torch.empty(0, 2, 64, device="cuda", dtype=BF16)
    i = torch.empty(0, dtype=torch.int64, device="cuda")
    assert aqd.qk_norm_rope(e, e, i, freqs(64)).q.shape == (0, 2, 64)
    aqd.cache_write(cache, e, e, i)
    assert aqd.cache_read(cache, i)[0].shape == (0, 2, 64)


def test_keys_alone_and_broadcast_inputs():
    q, k, v = inputs(10, 30, 4, 2, 64, BF16)
    pos, f = torch.arange(30, device="cuda"), freqs(64)
    want = aqd.qk_norm_rope(q, k, pos, f)
    none = aqd.qk_norm_rope(q[:, :0], k, pos, f)
    assert none.q.shape == (30, 0, 64) and torch.equal(none.k, want.k)
    one = q[:1, :1].expand(30, 4, 64)
    out = aqd.qk_norm_rope(one, k, pos, f, q_out=torch.empty(30, 4, 64, device="cuda", dtype=BF16)).q
    exact, size = rotated(one, None, pos, f, False, 0)
    close(out, exact, bound(exact, size, BF16))
    cache, slots = aqd.KVCache(4, 16, 2, 64), torch.arange(30, device="cuda")
    aqd.cache_write(cache, k[:, :1].expand(30, 2, 64), v, slots)
    gk, gv = aqd.cache_read(cache, slots)
    check_held(gk, k[:, :1].expand(30, 2, 64))
    check_held(gv, v)
