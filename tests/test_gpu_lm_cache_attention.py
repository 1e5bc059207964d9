"""Attention over the 4-bit cache against the formula in 64 bits on the cache's own values."""
import math

import pytest
import torch

from attention_ref import U, attended, close
from paper_2007_06919_gb300 import aqd

pytestmark = pytest.mark.gpu
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


class Case:
    """Sequences of given lengths in a cache of shuffled pages, the places behind their ends filled with NaN; queries of the last `asked` tokens."""

    def __init__(self, lens, asked, heads, kv, dim, page, dtype, seed=0, columns=0):
        torch.manual_seed(seed)
        pages = [-(-n // page) for n in lens]
        self.cache = aqd.KVCache(sum(pages) + 2, page, kv, dim)
        places = self.cache.pages * page
        loud = 1 + 2.0 * (torch.rand(kv, dim, device="cuda") < 0.1)
        k, v = (torch.randn(places, kv, dim, device="cuda") * loud + 0.3 * loud).to(dtype), torch.randn(places, kv, dim, device="cuda").to(dtype)
        order = torch.randperm(sum(pages), device="cuda").int() + 1
        self.table = torch.full((len(lens), max(columns, max(pages + [1]))), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
        at, self.slots = 0, []
        stale = torch.ones(places, dtype=torch.bool, device="cuda")
        for i, n in enumerate(pages):
            self.table[i, :n] = order[at:at + n]
            t = torch.arange(lens[i], device="cuda")
            self.slots.append(self.table[i].long()[t // page] * page + t % page)
            stale[self.slots[-1]] = False
            at += n
        k[stale], v[stale] = math.nan, math.nan
        aqd.cache_write(self.cache, k, v, torch.arange(places, device="cuda"))
        self.lens, self.asked = lens, asked
        self.lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
        at = [0]
        for n in asked:
            at.append(at[-1] + n)
        self.at = at
        self.starts = torch.tensor(at, dtype=torch.int32, device="cuda")
        self.q = torch.randn(at[-1], heads, dim, device="cuda").to(dtype)

    def want(self, scale, q=None):
        """(output, bound, lse, bound)."""
        q = self.q if q is None else q
        dim, dtype = q.shape[2], q.dtype
        o = torch.zeros_like(q, dtype=torch.float64)
        tol, e, et = o.clone(), o.new_zeros(o.shape[:2]), o.new_zeros(o.shape[:2])
        for i, n in enumerate(self.lens):
            a, b = self.at[i], self.at[i + 1]
            if a == b:
                continue
            k, v = aqd.cache_read(self.cache, self.slots[i], dtype=F32)
            o[a:b], e[a:b], mass, qsum = attended(q[a:b], k, v, [n - (b - a) + j + 1 for j in range(b - a)], scale)
            if n == 0:
                continue
            # a score: sums of dim products of |q| and 64 + code in float32, whose matrix instructions may cut instead of round (2^-22 of the
            # largest partial sum for each of dim / 16, and a few more steps), times the step; lowest value times sum |q| alike
            size = (k.amax(-1) - k.amin(-1)).max().item() / 15 * 79 + k.abs().max().item()
            score = scale * qsum * size * (dim / 16 + 6) * 2.0 ** -22 + 2.0 ** -22
            vmax, step = v.abs().max().item(), (v.amax(-1) - v.amin(-1)).max().item() / 15
            # output: weights off by the score's error in the sum and its normalizer; weights times step rounded to float16, times codes of up to 8 of
            # it; sums in float32
            tol[a:b] = (2 * score * vmax + 2.0 ** -11 * 8.2 * step + 2.0 ** -18 * (vmax + 8 * step))[..., None] + U[dtype] * o[a:b].abs()
            et[a:b] = score + 2.0 ** -22 * (1 + e[a:b].abs())
        return o, tol + 1e-30, e, et + 1e-30

    def run(self, **more):
        starts = None if all(n == 1 for n in self.asked) else self.starts
        return aqd.cache_attention(self.q, self.cache, self.table, self.lengths, starts=starts, **more)


LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 200, 255, 256, 257, 1000, 2049]


@pytest.mark.parametrize("heads,kv,dim,page,dtype", [(8, 2, 128, 64, BF16), (8, 1, 64, 16, F16), (3, 3, 192, 32, BF16), (10, 2, 256, 128, F16), (12, 1, 128, 16, BF16),
                                                     (40, 2, 64, 256, BF16), (1, 1, 128, 1024, F16), (20, 1, 256, 16, BF16)])
def test_one_token_of_each_sequence(heads, kv, dim, page, dtype):
    c = Case(LENS, [1] * len(LENS), heads, kv, dim, page, dtype)
    o, tol, e, et = c.want(dim ** -0.5)
    got, lse = c.run(lse=True)
    close(got, o, tol)
    close(lse, e, et)
    assert (got[0] == 0).all() and (lse[0] == -math.inf).all()
    assert aqd.device_status() == 0


@pytest.mark.parametrize("heads,kv,dim,page,dtype", [(8, 2, 128, 64, BF16), (28, 4, 64, 16, F16), (2, 2, 192, 32, BF16), (5, 1, 128, 16, BF16), (6, 1, 256, 16, F16)])
def test_several_tokens(heads, kv, dim, page, dtype):
    lens = [5, 3, 0, 700, 64, 2, 1, 33, 1500, 90, 40]
    asked = [2, 5, 2, 4, 0, 2, 1, 33, 7, 16, 3]  # more queries than places among them: the first ones see nothing
    c = Case(lens, asked, heads, kv, dim, page, dtype, seed=1)
    o, tol, e, et = c.want(0.11)
    got, lse = c.run(scale=0.11, lse=True)
    close(got, o, tol)
    close(lse, e, et)
    assert (got[c.at[1]:c.at[1] + 2] == 0).all() and (got[c.at[2]:c.at[3]] == 0).all()


@pytest.mark.parametrize("n,dim,kv", [(70_001, 128, 1), (30_000, 64, 2), (9000, 256, 1)])
def test_a_long_cache(n, dim, kv):
    c = Case([n, 5], [1, 1], 4 * kv, kv, dim, 64, F16, seed=2)
    o, tol, e, et = c.want(dim ** -0.5)
    got, lse = c.run(lse=True)
    close(got, o, tol)
    close(lse, e, et)


def test_many_sequences_of_uneven_lengths():
    torch.manual_seed(3)
    lens = [int(x) for x in torch.randint(0, 40, (700,))]
    lens[350] = 6000
    c = Case(lens, [1] * 700, 4, 2, 64, 16, BF16, seed=3)
    o, tol, e, et = c.want(0.125)
    got, lse = c.run(lse=True)
    close(got, o, tol)
    close(lse, e, et)


# Few sequences and heads: one, two, four or eight blocks join a row; longer tables split it among all. Without a place, with one, and with fewer steps than warps.
@pytest.mark.parametrize("lens,asked,heads,kv,dim,dtype", [([1024], [1], 8, 8, 128, BF16), ([8192, 1, 0], [1, 1, 1], 12, 3, 64, F16), ([700, 300, 2, 0], [3, 5, 4, 1], 14, 2, 64, BF16),
                                                           ([2000], [9], 6, 1, 192, F16), ([4096, 33], [1, 1], 20, 1, 256, BF16), ([513] * 19, [1] * 19, 16, 8, 128, F16),
                                                           ([8193, 8193], [1, 1], 4, 1, 128, BF16), ([3000] * 9, [2] * 9, 8, 1, 128, F16)])
def test_few_rows_in_several_blocks(lens, asked, heads, kv, dim, dtype):
    c = Case(lens, asked, heads, kv, dim, 64, dtype, seed=13)
    o, tol, e, et = c.want(dim ** -0.5)
    for _ in range(2):
        got, lse = c.run(lse=True)
        close(got, o, tol)
        close(lse, e, et)
    assert aqd.device_status() == 0


# (a warp looks through up to 128 sequences by itself; a block looks through more together)
@pytest.mark.parametrize("count", [31, 33, 128, 129, 257])
@pytest.mark.parametrize("longest", [100, 5000])
def test_any_number_of_sequences(count, longest):
    lens = [(7 * i) % 90 for i in range(count)]
    lens[count // 2] = longest
    c = Case(lens, [1 + i % 2 for i in range(count)], 4, 1, 64, 16, BF16, seed=14)
    o, tol, e, et = c.want(0.125)
    got, lse = c.run(lse=True)
    close(got, o, tol)
    close(lse, e, et)


def test_strides_and_rows_left_as_they_were():
    c = Case([100, 40, 300], [3, 1, 2], 6, 2, 128, 32, BF16, seed=4)
    want = c.run()
    wide = torch.zeros(6 + 4, 9, 136, device="cuda", dtype=BF16)
    q = wide[:10, 1:7, 3:131]
    q[:6] = c.q
    table = torch.cat([c.table, c.table], 1)[:, :c.table.shape[1]]
    out = torch.full((6, 12, 128), 5.0, device="cuda", dtype=BF16)  # heads outside tokens
    got = aqd.cache_attention(q, c.cache, table, c.lengths, starts=c.starts, out=out[:, 1:11].transpose(0, 1))
    assert torch.equal(got[:6], want) and (got[6:] == 5).all() and (out[:, 0] == 5).all() and (out[:, 11] == 5).all()


def test_masked_nan_and_pages_that_are_not_there():
    c = Case([64, 70], [2, 1], 4, 2, 64, 16, BF16, seed=5)
    want = c.run()
    # the last place, which the first of two queries does not see, holds NaN
    bad = torch.full((1, 2, 64), math.nan, device="cuda", dtype=BF16)
    k, v = aqd.cache_read(c.cache, c.slots[0][-1:])
    for which in ((bad, v), (k, bad)):
        aqd.cache_write(c.cache, *which, c.slots[0][-1:])
        got = c.run()
        assert torch.equal(got[0], want[0]) and got[1].isnan().all() and torch.equal(got[2], want[2])
    # two pages of the second sequence are none: as if its places there did not exist
    c.table[1, 1], c.table[1, 3] = -1, c.cache.pages
    t = torch.arange(70, device="cuda")
    seen = c.slots[1][((t // 16) != 1) & ((t // 16) != 3)]
    k, v = aqd.cache_read(c.cache, seen, dtype=F32)
    o, _, mass, _ = attended(c.q[2:], k, v, [seen.numel()], 0.125)
    got = c.run()
    close(got[2:], o, U[BF16] * o.abs() + 0.01 * mass)


def test_lengths_beyond_the_table_and_below_zero():
    c = Case([64, 30, 20], [1, 1, 1], 2, 1, 64, 16, BF16, seed=6)
    want = c.run()
    c.lengths = torch.tensor([2 ** 31 - 1, -5, 20], dtype=torch.int32, device="cuda")
    got = c.run()
    assert torch.equal(got[0], want[0]) and (got[1] == 0).all() and torch.equal(got[2], want[2])


def test_queries_of_any_size():
    c = Case([300], [1], 8, 1, 128, 32, BF16, seed=7)
    c.q[0, 0] = 0
    c.q[0, 1] *= 1e30
    c.q[0, 2] *= 1e-30
    c.q[0, 3, 5] = math.nan
    c.q[0, 4, 5] = math.inf
    got = c.run(scale=0.1)
    assert got[0, 3].isnan().all() and got[0, 4].isnan().all()
    rows = [0, 2, 5, 6, 7]
    o, tol, _, _ = c.want(0.1)
    close(got[0, rows], o[0, rows], tol[0, rows])
    assert got[0, 1].isfinite().all()


def test_value_steps_of_very_different_size():
    c = Case([200], [1], 4, 1, 64, 16, BF16, seed=8)
    k, v = aqd.cache_read(c.cache, c.slots[0])
    v = v * torch.logspace(-3, 3, 200, device="cuda").flip(0).to(BF16)[:, None, None]
    v[10], v[11] = 0, 2.0
    aqd.cache_write(c.cache, k, v.contiguous(), c.slots[0])
    o, tol, _, _ = c.want(0.125)
    close(c.run(), o, tol)
    v[:] = 0
    aqd.cache_write(c.cache, k, v, c.slots[0])
    assert (c.run() == 0).all()


def test_same_results_every_time_and_in_a_graph():
    c = Case([1000, 37, 5000, 1], [1] * 4, 8, 2, 128, 64, BF16, seed=9)
    want, lse = c.run(lse=True)
    for _ in range(3):
        got, e = c.run(lse=True)
        assert torch.equal(got, want) and torch.equal(e, lse)
    spaces = [aqd.cache_attention_workspace(c.q, c.cache, 4) for _ in range(2)]
    outs = [torch.empty_like(c.q) for _ in range(2)]
    graphs = []
    torch.cuda.synchronize()
    for w, o in zip(spaces, outs):
        w.fill_(255)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            aqd.cache_attention(c.q, c.cache, c.table, c.lengths, out=o, workspace=w)
        graphs.append(g)
    c.lengths.copy_(torch.tensor([900, 30, 4000, 1], dtype=torch.int32))  # the graphs read lengths as they are when they run
    want = c.run()
    streams = [torch.cuda.Stream() for _ in graphs]
    torch.cuda.synchronize()
    for g, s in zip(graphs, streams):
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, want)


def test_on_another_stream():
    c = Case([300, 4000], [1, 1], 8, 2, 64, 16, F16, seed=10)
    want = c.run()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = c.run(stream=s)
    s.synchronize()
    assert torch.equal(got, want)


def test_no_sequences():
    c = Case([10], [1], 2, 1, 64, 16, BF16)
    out = torch.full((3, 2, 64), 4.0, device="cuda", dtype=BF16)
    none = torch.zeros(1, dtype=torch.int32, device="cuda")
    aqd.cache_attention(out.clone(), c.cache, c.table[:0], c.lengths[:0], starts=none, out=out)
    assert (out == 4).all()


def test_pages_of_more_than_32_bits():
    kv, dim = 65535, 64
    cache = aqd.KVCache(2, 1024, kv, dim)
    assert cache.data.numel() // 2 > 1 << 32
    torch.manual_seed(11)
    n = 20
    k, v = (torch.randn(n, kv, dim, device="cuda", dtype=BF16) for _ in range(2))
    slots = torch.arange(n, device="cuda") + 1024
    aqd.cache_write(cache, k, v, slots)
    q = torch.randn(1, kv, dim, device="cuda", dtype=BF16)
    for columns in (1, 2):  # a block for each head, and runs
        table = torch.full((1, columns), 1, dtype=torch.int32, device="cuda")
        got = aqd.cache_attention(q, cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"))
        ck, cv = aqd.cache_read(cache, slots, dtype=F32)
        p = (torch.einsum("hd,mhd->hm", q[0].double(), ck.double()) / 8).softmax(1)
        want = torch.einsum("hm,mhd->hd", p, cv.double())
        # (the sums of the scores' and weights' bounds above, for values of 5 and steps of 0.6)
        close(got[0], want, 0.02 + U[BF16] * want.abs())


def test_broadcast_queries():
    c = Case([90, 33], [1, 1], 6, 2, 64, 16, BF16, seed=12)
    c.q = c.q[:, :1].expand(2, 6, 64)
    o, tol, _, _ = c.want(0.125)
    close(aqd.cache_attention(c.q, c.cache, c.table, c.lengths, out=torch.empty(2, 6, 64, device="cuda", dtype=BF16)), o, tol)
