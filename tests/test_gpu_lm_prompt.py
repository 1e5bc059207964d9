"""Attention over packed prompts against the formula in 64 bits."""
import math

import pytest
import torch

from attention_ref import U, attended, close
from paper_2007_06919_gb300 import aqd

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


def starts_of(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at, torch.tensor(at, dtype=torch.int32, device="cuda")


def inputs(seed, tokens, kv_tokens, heads, kv, dim, dtype):
    torch.manual_seed(seed)
    q = torch.randn(tokens, heads, dim, device="cuda").to(dtype)
    k = (1.5 * torch.randn(kv_tokens, kv, dim, device="cuda")).to(dtype)
    v = torch.randn(kv_tokens, 2 * kv + heads, dim, device="cuda").to(dtype)[:, heads + kv:]
    return q, k, v


def reference(q, k, v, at, kat, causal, scale, rows=None):
    """(output, bound, lse, bound); rows: the tokens that are wanted."""
    dim, dtype = q.shape[2], q.dtype
    o = torch.zeros_like(q, dtype=torch.float64)
    tol, e, et = o.clone(), o.new_zeros(o.shape[:2]), o.new_zeros(o.shape[:2])
    for i in range(len(at) - 1):
        n, m = at[i + 1] - at[i], kat[i + 1] - kat[i]
        pick = [r for r in range(n) if rows is None or at[i] + r in rows]
        if not pick:
            continue
        x, kk, vv = q[at[i]:at[i + 1]][pick], k[kat[i]:kat[i + 1]], v[kat[i]:kat[i + 1]]
        see = [m - n + r + 1 if causal else m for r in pick]
        out, lse, mass, qsum = attended(x, kk, vv, see, scale)
        r = [at[i] + j for j in pick]
        o[r], e[r] = out, lse
        # a score: dim products of float32 sums, cut at 2^-22 of the largest partial sum for each of dim / 16 steps; weights rounded to the type; output rounded
        score = scale * qsum * (kk.abs().max().item() if m else 0.0) * (dim / 16 + 6) * 2.0 ** -22 + 2.0 ** -21
        vmax = vv.abs().max().item() if m else 0.0
        tol[r] = U[dtype] * (out.abs() + mass) * 1.01 + (2 * score * vmax)[..., None] + 1e-30
        et[r] = score + 2.0 ** -22 * lse.abs().nan_to_num(0.0, 0.0, 0.0)
    return o, tol, e, et


LENS = [1, 2, 63, 64, 65, 127, 128, 129, 0, 200, 255, 256, 257, 300, 31]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv,dim,dtype", [(4, 2, 128, BF16), (3, 1, 64, F16), (2, 2, 192, BF16), (2, 1, 256, F16), (7, 7, 64, BF16), (8, 1, 128, F16)])
def test_packed_prompts(heads, kv, dim, dtype, causal):
    at, starts = starts_of(LENS)
    q, k, v = inputs(dim + heads, at[-1], at[-1], heads, kv, dim, dtype)
    o, tol, e, et = reference(q, k, v, at, at, causal, dim ** -0.5)
    got, lse = aqd.prompt_attention(q, k, v, starts, causal=causal, lse=True)
    close(got, o, tol)
    close(lse, e, et)
    assert aqd.device_status() == 0


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim,dtype", [(128, BF16), (64, F16), (192, F16), (256, BF16)])
def test_other_keys_than_queries(dim, dtype, causal):
    """A prompt that goes on from earlier tokens, and queries before the first key, which see nothing."""
    lens, klens = [5, 100, 1, 64, 0, 40, 7, 300], [500, 100, 700, 10, 30, 0, 7, 40]
    at, starts = starts_of(lens)
    kat, kstarts = starts_of(klens)
    q, k, v = inputs(dim, at[-1], kat[-1], 4, 2, dim, dtype)
    o, tol, e, et = reference(q, k, v, at, kat, causal, 0.2)
    got, lse = aqd.prompt_attention(q, k, v, starts, kv_starts=kstarts, causal=causal, scale=0.2, lse=True)
    close(got, o, tol)
    close(lse, e, et)
    assert (got[at[5]:at[6]] == 0).all() and (lse[at[5]:at[6]] == -math.inf).all()
    if causal:
        assert (got[at[3]:at[3] + 54] == 0).all()


@pytest.mark.parametrize("n,dim,dtype", [(5000, 128, BF16), (3001, 64, F16), (1500, 256, BF16)])
def test_long_prompts(n, dim, dtype):
    at, starts = starts_of([7, n, 1])
    q, k, v = inputs(n, at[-1], at[-1], 2, 1, dim, dtype)
    rows = set(range(0, 20)) | {7 + r for r in (255, 256, 1023, 1024, n - 257, n - 129, n - 2, n - 1)} | {7 + n}
    o, tol, e, et = reference(q, k, v, at, at, True, dim ** -0.5, rows)
    got, lse = aqd.prompt_attention(q, k, v, starts, lse=True)
    r = sorted(rows)
    close(got[r], o[r], tol[r])
    close(lse[r], e[r], et[r])


def test_large_scores():
    """Scores far apart: maxima that grow from tile to tile, weights that vanish."""
    at, starts = starts_of([600, 100])
    q, k, v = inputs(1, 700, 700, 2, 2, 128, BF16)
    k = k * torch.linspace(0.1, 20, 700, device="cuda").to(BF16)[:, None, None]
    o, tol, e, et = reference(q, k, v, at, at, True, 0.3)
    got, lse = aqd.prompt_attention(q, k, v, starts, scale=0.3, lse=True)
    close(got, o, tol)
    close(lse, e, et)


@pytest.mark.parametrize("dim", [64, 128, 192])
def test_strides_and_rows_left_as_they_were(dim):
    at, starts = starts_of([100, 3, 260])
    q, k, v = inputs(2, 363, 363, 4, 2, dim, BF16)
    want = aqd.prompt_attention(q, k, v, starts)
    wide = torch.full((4, 370, dim + 8), math.nan, device="cuda", dtype=BF16)
    wide[:, :363, :dim] = q.transpose(0, 1)
    out = torch.full((370, 4, dim + 24), 5.0, device="cuda", dtype=BF16)
    kk = torch.cat([k, torch.full((7, 2, dim), math.nan, device="cuda", dtype=BF16)])
    vv = torch.cat([v, torch.full((7, 2, dim), math.nan, device="cuda", dtype=BF16)])
    aqd.prompt_attention(wide[:, :, :dim].transpose(0, 1), kk, vv, starts, out=out[:, :, 8:8 + dim])
    assert torch.equal(out[:363, :, 8:8 + dim], want) and (out[363:] == 5).all() and (out[..., :8] == 5).all() and (out[..., 8 + dim:] == 5).all()


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_nan_and_infinity_stay_in_their_sequence(dim):
    lens = [130, 70, 200, 256, 65]
    at, starts = starts_of(lens)
    q, k, v = inputs(3, at[-1], at[-1], 2, 1, dim, F16)
    want, lse = aqd.prompt_attention(q, k, v, starts, lse=True)
    for bad in (math.nan, math.inf):
        qq, kk, vv = q.clone(), k.clone(), v.clone()
        kk[at[1]:at[2]] = bad
        vv[at[1]:at[2]] = bad
        qq[at[1]:at[2]] = bad
        kk[at[3] + 255], vv[at[3] + 255] = bad, bad  # the last of a sequence: seen by its last query alone
        got, e = aqd.prompt_attention(qq, kk, vv, starts, lse=True)
        keep = torch.ones(at[-1], dtype=torch.bool, device="cuda")
        keep[at[1]:at[2]] = False
        keep[at[3]:at[4]] = False
        assert torch.equal(got[keep], want[keep]) and torch.equal(e[keep], lse[keep])
        assert not got[at[1]:at[2]].isfinite().any()
        assert not got[at[4] - 1].isfinite().all(-1).any()


def test_key_nan_that_no_query_of_a_tile_sees():
    at, starts = starts_of([300])
    q, k, v = inputs(4, 300, 300, 2, 2, 64, BF16)
    want = aqd.prompt_attention(q, k, v, starts)
    k[290] = math.nan  # scores alone: queries before it are as they were
    got = aqd.prompt_attention(q, k, v, starts)
    assert torch.equal(got[:290], want[:290]) and got[290:].isnan().all()


def test_same_results_every_time_in_a_graph_and_on_another_stream():
    at, starts = starts_of([500, 77, 1000])
    q, k, v = inputs(5, at[-1], at[-1], 4, 2, 128, BF16)
    want = aqd.prompt_attention(q, k, v, starts)
    for _ in range(3):
        assert torch.equal(aqd.prompt_attention(q, k, v, starts), want)
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        aqd.prompt_attention(q, k, v, starts, out=out)
    out.zero_()
    g.replay()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    got = aqd.prompt_attention(q, k, v, starts, stream=s)
    s.synchronize()
    assert torch.equal(got, want)


def test_no_sequences():
    q, k, v = inputs(6, 3, 3, 2, 2, 64, BF16)
    out = torch.full_like(q, 4.0)
    aqd.prompt_attention(q, k, v, torch.zeros(1, dtype=torch.int32, device="cuda"), out=out)
    assert (out == 4).all()
    assert aqd.prompt_attention(q[:0], k[:0], v[:0], torch.zeros(3, dtype=torch.int32, device="cuda")).shape == (0, 2, 64)


@pytest.mark.parametrize("dim", [64, 128])
def test_broadcast_keys_and_two_calls_at_once(dim):
    at, starts = starts_of([300, 41])
    q, k, v = inputs(7, 341, 341, 4, 2, dim, BF16)
    k = k[:, :1].expand(341, 2, dim)
    o, tol, _, _ = reference(q, k, v, at, at, True, dim ** -0.5)
    close(aqd.prompt_attention(q, k, v, starts), o, tol)
    k = k.contiguous()
    want = aqd.prompt_attention(q, k, v, starts)
    close(want, o, tol)
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    torch.cuda._sleep(2_000_000)
    got = [aqd.prompt_attention(q, k, v, starts, stream=s) for s in streams for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)


def test_many_short_prompts():
    """More jobs than blocks, most of them a row or two; sequences without queries and without keys among them."""
    torch.manual_seed(8)
    lens = [int(n) for n in torch.randint(0, 5, (900,))]
    klens = [int(n) for n in torch.randint(0, 7, (900,))]
    lens[450], klens[450] = 700, 900
    at, starts = starts_of(lens)
    kat, kstarts = starts_of(klens)
    q, k, v = inputs(9, at[-1], kat[-1], 2, 1, 64, F16)
    for causal in (True, False):
        o, tol, e, et = reference(q, k, v, at, kat, causal, 0.125)
        got, lse = aqd.prompt_attention(q, k, v, starts, kv_starts=kstarts, causal=causal, lse=True)
        close(got, o, tol)
        close(lse, e, et)
    assert aqd.device_status() == 0


# Heads of 192 and 256 have a kernel of their own: one to many steps, tiles that end in a sequence, maxima that grow, weights that vanish.
@pytest.mark.parametrize("dim,dtype", [(192, BF16), (256, F16), (192, F16), (256, BF16)])
def test_wide_heads(dim, dtype):
    lens = [1, 128, 129, 256, 257, 383, 384, 385, 640, 2000]
    at, starts = starts_of(lens)
    q, k, v = inputs(10 + dim, at[-1], at[-1], 3, 1, dim, dtype)
    for scale, ramp in ((dim ** -0.5, False), (0.25, True)):
        kk = k * torch.linspace(0.1, 15, at[-1], device="cuda").to(dtype)[:, None, None] if ramp else k
        o, tol, e, et = reference(q, kk, v, at, at, True, scale)
        for _ in range(2):
            got, lse = aqd.prompt_attention(q, kk, v, starts, scale=scale, lse=True)
            close(got, o, tol)
            close(lse, e, et)
    assert aqd.device_status() == 0


@pytest.mark.parametrize("dim", [192, 256])
def test_wide_heads_of_many_short_prompts_broadcast_and_at_once(dim):
    torch.manual_seed(11)
    lens = [int(n) for n in torch.randint(0, 4, (400,))]
    klens = [int(n) for n in torch.randint(0, 6, (400,))]
    lens[200], klens[200] = 500, 700
    at, starts = starts_of(lens)
    kat, kstarts = starts_of(klens)
    q, k, v = inputs(12, at[-1], kat[-1], 4, 2, dim, BF16)
    for causal in (True, False):
        o, tol, e, et = reference(q, k, v, at, kat, causal, 0.08)
        got, lse = aqd.prompt_attention(q, k, v, starts, kv_starts=kstarts, causal=causal, scale=0.08, lse=True)
        close(got, o, tol)
        close(lse, e, et)
    want = got
    streams = [torch.cuda.Stream() for _ in range(4)]
    torch.cuda.synchronize()
    torch.cuda._sleep(2_000_000)
    runs = [aqd.prompt_attention(q, k, v, starts, kv_starts=kstarts, causal=False, scale=0.08, stream=s) for s in streams for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in runs)
    k = k[:, :1].expand(-1, 2, -1)  # (a stride of zero: the other kernel)
    o, tol, _, _ = reference(q, k, v, at, kat, True, 0.08)
    close(aqd.prompt_attention(q, k, v, starts, kv_starts=kstarts, scale=0.08), o, tol)
    assert aqd.device_status() == 0
