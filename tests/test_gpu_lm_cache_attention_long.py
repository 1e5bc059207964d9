"""Attention over long caches: warps whose runs go round their rings and past 32 steps, parts joined from few and many blocks, each judged by the error of whole rows."""
import pytest
import torch

from attention_ref import attended
from paper_2007_06919_gb300 import aqd
from test_gpu_lm_cache_attention import Case

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
STAGES = {64: 6, 128: 3, 192: 4, 256: 3}


def runs(c, heads, kv):
    """(steps of the longest run, most runs of a sequence's tile): how a call's work is split. A step is 32 places; as many runs as fill 152 SMs once, in even lengths."""
    group, dim, tokens, seqs = heads // kv, c.q.shape[2], c.q.shape[0], len(c.lens)
    two = dim <= 128 and tokens * group > 8 * seqs
    rows, warps = (16 if two else 8), 152 * 8 * (1 if two or dim > 128 else 2)
    tiles = [-(-n * group // rows) for n in c.asked]
    steps = [-(-n // 32) for n in c.lens]
    most = warps - sum(tiles) * kv if sum(tiles) * kv < warps // 2 else warps // 2
    ratio = most / max(1, sum(t * s for t, s in zip(tiles, steps)) * kv)
    split = [max(1, min(s, -int(-s * ratio // 1))) for s in steps]
    return max(-(-s // r) for s, r in zip(steps, split)), max(split)


def error(got, want):
    """The largest error of a row's output, relative to the row's size."""
    return ((got.double() - want).norm(dim=-1) / want.norm(dim=-1)).max().item()


# Half a step of an output's rounding at random is u / sqrt(3) of a row, u = 2^-11 or 2^-8; so are the weights' roundings to float16 (2^-11), whose errors add up
# as the values themselves do; scores are off by some 2^-13 (dim products of float32 sums, cut): together below 2^-11 (1 / 3 + 1 / 3 + 1 / 16)^(1/2) = 4.2e-4 and, in
# bfloat16, 2.3e-3. About twice that is the bound. The logarithm of the sum is off by the scores' mean error: each is at most 3e-3 off if every partial sum of q . (64 + n)
# were as large as that of |q| 79, which signs at random make a tenth; below 1e-3. A part left out, one of n, is an error of n^(-1/2) of a row
# (less where values have a mean). Outputs without a part have to be off by 1.5 bounds: then a kernel that lost it, itself at most half a bound off as above, fails.
BOUND = {F16: 1e-3, BF16: 5e-3}


@pytest.mark.parametrize("lens,asked,heads,kv,dim,page,dtype", [
    ([8192] * 12 + [5, 0, 31, 9000], 1, 32, 8, 128, 64, F16),                    # 12 steps a warp
    ([20_480] * 16, 1, 32, 8, 128, 64, F16),                                     # 36
    ([30_000, 20_001, 25_000, 70, 33_333] * 4, 1, 16, 8, 64, 16, F16),           # 48
    ([16_400, 12_000, 100] * 7, 1, 8, 8, 192, 32, F16),                          # 47
    ([10_240] * 17, 1, 4, 4, 256, 64, BF16),                                     # 19
    ([20_000, 17, 21_000] * 4, 1, 8, 8, 256, 16, F16),                           # 37
    ([12_345, 9000, 40_000] * 5, 3, 32, 4, 128, 16, F16),                        # 70, 16 rows a task
    ([7000 + 13 * i for i in range(300)], 1, 8, 2, 64, 16, F16),                 # 92, and a block looks the tasks up together
])
def test_runs_that_go_round_the_ring(lens, asked, heads, kv, dim, page, dtype):
    c = Case(lens, [min(asked, n) if asked > 1 else 1 for n in lens], heads, kv, dim, page, dtype, seed=20)
    steps, _ = runs(c, heads, kv)
    assert steps > STAGES[dim] + 3
    got, lse = c.run(lse=True)
    again, _ = c.run(lse=True)
    assert torch.equal(got, again)
    for i in sorted({0, 1, len(lens) // 2, len(lens) - 2, len(lens) - 1}):
        a, b = c.at[i], c.at[i + 1]
        if lens[i] == 0:
            assert (got[a:b] == 0).all()
            continue
        k, v = aqd.cache_read(c.cache, c.slots[i], dtype=F32)
        see = [lens[i] - (b - a) + j + 1 for j in range(b - a)]
        o, e, _, _ = attended(c.q[a:b], k, v, see, dim ** -0.5)
        assert error(got[a:b], o) <= BOUND[dtype]
        assert (lse[a:b].double() - e).abs().max() <= 1e-3
        if lens[i] > 1000:  # what the bound would say of an output without a warp's run, and of none
            less, _, _, _ = attended(c.q[a:b], k[32 * steps:], v[32 * steps:], [n - 32 * steps for n in see], dim ** -0.5)
            assert error(less, o) > 1.5 * BOUND[dtype] and error(torch.zeros_like(o), o) > 0.9
    assert aqd.device_status() == 0


def test_runs_of_more_than_32_steps_are_among_them():
    """(Page numbers are looked up 32 steps at a time.)"""
    for lens, heads, kv, dim, tokens in (([20_480] * 16, 32, 8, 128, 1), ([30_000, 20_001, 25_000, 70, 33_333] * 4, 16, 8, 64, 1), ([16_400, 12_000, 100] * 7, 8, 8, 192, 1),
                                         ([20_000, 17, 21_000] * 4, 8, 8, 256, 1)):
        from types import SimpleNamespace
        c = SimpleNamespace(lens=lens, asked=[1] * len(lens), q=torch.empty(len(lens), heads, dim))
        assert runs(c, heads, kv)[0] > 33


@pytest.mark.parametrize("n,heads,kv,dim,dtype", [(70_001, 4, 1, 128, F16), (200_001, 16, 2, 128, F16), (30_000, 8, 2, 64, F16), (9000, 4, 1, 256, F16), (120_000, 12, 1, 64, F16),
                                                  (50_000, 5, 1, 192, F16), (400_000, 1, 1, 64, BF16)])
def test_parts_joined_from_many_blocks(n, heads, kv, dim, dtype):
    """Each part's weight in the output and in the logarithm: values whose mean changes along the cache, and one part's share above the bounds."""
    c = Case([n, 5], [1, 1], heads, kv, dim, 64, dtype, seed=21)
    # each eighth of the sequence has values of another mean
    k, v = aqd.cache_read(c.cache, c.slots[0])
    v = (v.float() + 0.3 * torch.randn(8, kv, dim, device="cuda")[torch.arange(n, device="cuda") * 8 // n]).to(v.dtype)
    aqd.cache_write(c.cache, k, v, c.slots[0])
    _, parts = runs(c, heads, kv)
    blocks = -(-parts // 8)
    k, v = aqd.cache_read(c.cache, c.slots[0], dtype=F32)
    o, e, _, _ = attended(c.q[:1], k, v, [n], dim ** -0.5)
    got, lse = c.run(lse=True)
    assert error(got[:1], o) <= BOUND[dtype] and (lse[:1].double() - e).abs().max() <= 1e-3
    piece = n // blocks
    for at in (0, n // 2, n - piece):
        seen = torch.ones(n, dtype=torch.bool, device="cuda")
        seen[at:at + piece] = False
        less, el, _, _ = attended(c.q[:1], k[seen], v[seen], [n], dim ** -0.5)
        assert error(less, o) > 1.5 * BOUND[dtype] and (el - e).abs().min() > 2e-3


# A warp looks through up to 32 sequences by itself, the 256 threads of a block through more, 256 at a time.
@pytest.mark.parametrize("count", [32, 33, 255, 256, 257, 512, 513])
@pytest.mark.parametrize("longest", [100, 6000])
def test_sequences_around_the_look_up(count, longest):
    lens = [1 + (7 * i) % 90 for i in range(count)]
    lens[count - 1] = longest
    c = Case(lens, [1] * count, 4, 1, 64, 16, F16, seed=22)
    got = c.run()
    for i in sorted({0, 31, count // 2, count - 2, count - 1}):
        k, v = aqd.cache_read(c.cache, c.slots[i], dtype=F32)
        o, _, _, _ = attended(c.q[i:i + 1], k, v, [lens[i]], 0.125)
        assert error(got[i:i + 1], o) <= BOUND[F16]
