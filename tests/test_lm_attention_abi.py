"""CPU checks of the attention operators' C entry points and binding: what they refuse before a launch (the device addresses below are never
read), sizes, and the packed structs."""
import ctypes

import pytest
import torch

from paper_2007_06919_gb300 import aqd, build
from test_lm_host_checks import Tensor, made  # noqa: F401

A = 0x7000_0000_0000  # an address no call may read
F32, F16, BF16, I32 = range(4)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return aqd._calls()


def cache(data=A, pages=10, page=64, kv=2, dim=128):
    return aqd._KV_CACHE.pack(data, pages, page, kv, dim)


def rope(n=4, h=8, kv=2, d=128, dt=BF16, q=A, lq=1024, lqh=128, k=A, lk=256, lkh=128, v=A, lv=256, lvh=128, qo=A + 64, lqo=1024, lqoh=128, ko=A + 64, lko=256, lkoh=128,
         wq=A, wk=A, wd=BF16, eps=1e-6, pos=A, f=A, rot=128, inter=0, slots=A):
    return aqd._QK_ROPE.pack(n, h, kv, d, dt, q, lq, lqh, k, lk, lkh, v, lv, lvh, qo, lqo, lqoh, ko, lko, lkoh, wq, wk, wd, eps, pos, f, rot, inter, slots)


def rows(n=4, dt=BF16, k=A, lk=256, lkh=128, v=A, lv=256, lvh=128, slots=A):
    return aqd._CACHE_ROWS.pack(n, dt, k, lk, lkh, v, lv, lvh, slots)


def attn(n=4, seqs=4, h=8, dt=BF16, scale=0.1, q=A, lq=1024, lqh=128, o=A, lo=1024, loh=128, lse=0, starts=0, lens=A, table=A, lt=8, cols=8):
    return aqd._CACHE_ATTENTION.pack(n, seqs, h, dt, scale, q, lq, lqh, o, lo, loh, lse, starts, lens, table, lt, cols)


def prompt(n=40, nk=40, seqs=2, h=8, kv=2, d=128, dt=BF16, causal=1, scale=0.1, q=A, lq=1024, lqh=128, k=A, lk=256, lkh=128, v=A, lv=256, lvh=128, o=A, lo=1024, loh=128,
           lse=0, starts=A, ks=0):
    return aqd._PROMPT.pack(n, nk, seqs, h, kv, d, dt, causal, scale, q, lq, lqh, k, lk, lkh, v, lv, lvh, o, lo, loh, lse, starts, ks)


BAD_CACHES = [None, cache(data=0), cache(data=A + 16), cache(pages=0), cache(pages=1 << 31), cache(page=8), cache(page=48), cache(page=2048), cache(kv=0), cache(dim=96),
              cache(dim=32), cache(dim=320), cache(pages=1 << 30, page=1024)]


def test_cache_sizes(lib):
    f = lib.aqd_kv_cache_bytes
    assert f(1, 16, 1, 64) == 16 * 2 * (32 + 4) and f(10, 64, 8, 128) == 10 * 64 * 8 * 2 * (64 + 4)
    for a in ((0, 16, 1, 64), (1, 15, 1, 64), (1, 16, 0, 64), (1, 16, 1, 100), (-1, 16, 1, 64), (1 << 30, 1024, 8, 256), (1, 16, 70000, 64)):
        assert f(*a) == 0, a


def test_rotation_refuses(lib):
    f = lib.aqd_qk_norm_rope
    assert f(rope(n=0, q=0, k=0, qo=0, ko=0, pos=0, f=0), None, None) == 0
    for a in (None, rope(n=-1), rope(n=1 << 31), rope(h=-1), rope(h=70000), rope(kv=0), rope(d=0), rope(d=7), rope(d=514), rope(dt=I32), rope(dt=9), rope(q=0), rope(q=A + 1),
              rope(lq=-1), rope(lqh=-8), rope(k=0), rope(k=A + 1), rope(qo=0), rope(qo=A + 1), rope(lqo=1023), rope(lqoh=127), rope(lko=255), rope(ko=0), rope(wq=A + 1), rope(wd=I32),
              rope(eps=-1.0), rope(eps=float("nan")), rope(rot=-2), rope(rot=3), rope(rot=130), rope(pos=0), rope(f=0), rope(pos=A + 4), rope(f=A + 2),
              rope(qo=A, lqo=2048), rope(ko=A, lko=512)):
        assert f(a, None, None) == 1, a
    for c in BAD_CACHES[1:] + [cache(kv=4), cache(dim=64)]:
        assert f(rope(), c, None) == 1, c
    for a in (rope(v=0), rope(v=A + 1), rope(slots=0), rope(slots=A + 4), rope(lv=-1)):
        assert f(a, cache(), None) == 1, a


def test_cache_rows_refuse(lib):
    for f in (lib.aqd_cache_write, lib.aqd_cache_read):
        assert f(rows(n=0, k=0, v=0, slots=0), cache(), None) == 0
        for c in BAD_CACHES:
            assert f(rows(), c, None) == 1, c
        for a in (None, rows(n=-1), rows(n=1 << 31), rows(dt=I32), rows(k=A + 1), rows(lk=-1), rows(slots=0), rows(slots=A + 4), rows(v=A + 1)):
            assert f(a, cache(), None) == 1, a
    for a in (rows(k=0), rows(v=0)):
        assert lib.aqd_cache_write(a, cache(), None) == 1
    for a in (rows(k=0, v=0), rows(lk=255), rows(lkh=127), rows(lv=0, lvh=0)):
        assert lib.aqd_cache_read(a, cache(), None) == 1


def test_cache_attention_refuses(lib):
    f, size = lib.aqd_cache_attention, lib.aqd_cache_attention_workspace_bytes
    need = size(4, 4, 8, cache())
    assert need > 0 and f(attn(n=0, seqs=0, q=0, o=0), cache(), None, 0, None) == 0
    assert f(attn(n=0, seqs=3, q=0, o=0, starts=A), cache(), None, 0, None) == 0
    for a in (None, attn(n=-1), attn(n=1 << 31), attn(seqs=-1), attn(n=5), attn(h=0), attn(h=7), attn(h=70000), attn(dt=F32), attn(scale=0.0), attn(scale=-1.0), attn(scale=float("inf")),
              attn(q=0), attn(q=A + 1), attn(lq=-1), attn(o=0), attn(lo=1000), attn(loh=64), attn(lens=0), attn(lens=A + 2), attn(table=0), attn(table=A + 1), attn(lt=7), attn(cols=-1),
              attn(cols=1 << 26, lt=1 << 26), attn(lse=A + 2), attn(starts=A + 2)):
        assert f(a, cache(), A, need, None) == 1, a
    for c in BAD_CACHES:
        assert f(attn(), c, A, need, None) == 1, c
    assert f(attn(), cache(), None, need, None) == 1 and f(attn(), cache(), A + 16, need, None) == 1 and f(attn(), cache(), A, need - 1, None) == 1
    for a in ((-1, 4, 8, cache()), (4, -1, 8, cache()), (4, 4, 7, cache()), (4, 4, 8, cache(dim=96)), (1 << 31, 4, 8, cache()), (1 << 28, 4, 8, cache())):
        assert size(*a) == 0, a


def test_prompt_refuses(lib):
    f = lib.aqd_prompt_attention
    assert f(prompt(n=0, q=0, o=0), None) == 0 and f(prompt(seqs=0, starts=0), None) == 0
    for a in (None, prompt(n=-1), prompt(n=1 << 31), prompt(nk=-1), prompt(nk=1 << 31), prompt(seqs=-1), prompt(h=0), prompt(kv=0), prompt(kv=3), prompt(d=96), prompt(d=0), prompt(dt=F32),
              prompt(scale=0.0), prompt(scale=float("nan")), prompt(q=0), prompt(q=A + 8), prompt(k=0), prompt(v=A + 2), prompt(o=0), prompt(o=A + 8), prompt(lq=1028), prompt(lkh=132),
              prompt(lv=-8), prompt(lo=1000), prompt(loh=120), prompt(starts=0), prompt(starts=A + 2), prompt(ks=A + 1), prompt(lse=A + 2)):
        assert f(a, None) == 1, a


def test_packed_structs_have_the_header_sizes():
    p, q, i, f = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float
    t = [p, q, q]
    for packed, fields in ((aqd._KV_CACHE, [p, q, i, i, i]), (aqd._QK_ROPE, [q, i, i, i, i] + 5 * t + [p, p, i, f, p, p, i, i, p]), (aqd._CACHE_ROWS, [q, i] + 2 * t + [p]),
                           (aqd._CACHE_ATTENTION, [q, i, i, i, f] + 2 * t + [p, p, p, p, q, i]), (aqd._PROMPT, [q, q] + 6 * [i] + [f] + 4 * t + [p, p, p])):
        c = type("S", (ctypes.Structure,), {"_fields_": [(f"f{n}", x) for n, x in enumerate(fields)]})
        assert packed.size == ctypes.sizeof(c)


# ------------------------------------------------------------------ the binding


def heads(n=4, h=8, d=128, dtype=torch.bfloat16, device=0, strides=None):
    return Tensor((n, h, d), dtype, device, strides)


def ints(n, dtype=torch.int64, device=0):
    return Tensor((n,), dtype, device)


def a_cache(device=0):
    c = aqd.KVCache.__new__(aqd.KVCache)
    c.pages, c.page_size, c.kv_heads, c.head_dim, c.index, c.desc = 10, 64, 2, 128, device, b""
    c.device = torch.device("cuda", device)
    return c


def table(device=0, seqs=4):
    return Tensor((seqs, 8), torch.int32, device)


CALLS = {
    "qk_norm_rope": lambda d, s: aqd.qk_norm_rope(heads(device=d), heads(h=2, device=d), ints(4, device=d), Tensor((64,), torch.float32, d), stream=s),
    "append": lambda d, s: aqd.qk_norm_rope(heads(device=d), heads(h=2, device=d), None, None, v=heads(h=2, device=d), cache=a_cache(d), slots=ints(4, device=d), stream=s),
    "cache_write": lambda d, s: aqd.cache_write(a_cache(d), heads(h=2, device=d), heads(h=2, device=d), ints(4, device=d), stream=s),
    "cache_read": lambda d, s: aqd.cache_read(a_cache(d), ints(4, device=d), stream=s),
    "cache_attention": lambda d, s: aqd.cache_attention(heads(device=d), a_cache(d), table(d), ints(4, torch.int32, d), workspace=Tensor((1 << 20,), torch.uint8, d), stream=s),
    "prompt_attention": lambda d, s: aqd.prompt_attention(heads(device=d), heads(h=2, device=d), heads(h=2, device=d), ints(3, torch.int32, d), stream=s),
}


@pytest.mark.parametrize("call", list(CALLS))
def test_tensors_and_streams_of_another_device_than_the_current_one(made, call):  # noqa: F811
    from types import SimpleNamespace
    here, there = (SimpleNamespace(device=torch.device("cuda", i), cuda_stream=5) for i in (0, 1))
    for d, s in ((1, None), (1, there), (0, there), (1, here)):
        with pytest.raises(ValueError, match="device"):
            CALLS[call](d, s)
    assert [n for n in made if not n.endswith("_bytes")] == []
    CALLS[call](0, None)
    CALLS[call](0, here)
    assert len([n for n in made if not n.endswith("_bytes")]) == 2


def test_what_does_not_fit_together(made):  # noqa: F811
    q, k = heads(), heads(h=2)
    p, f = ints(4), Tensor((64,), torch.float32)
    w = Tensor((128,), torch.bfloat16)
    c, slots = a_cache(), ints(4)
    for call in (lambda: aqd.qk_norm_rope(q, heads(n=5, h=2), p, f), lambda: aqd.qk_norm_rope(q, heads(h=2, d=64), p, f), lambda: aqd.qk_norm_rope(q, heads(h=2, dtype=torch.float16), p, f),
                 lambda: aqd.qk_norm_rope(q, k, None, f), lambda: aqd.qk_norm_rope(q, k, ints(5), f), lambda: aqd.qk_norm_rope(q, k, ints(4, torch.int32), f),
                 lambda: aqd.qk_norm_rope(q, k, p, Tensor((64,), torch.float64)), lambda: aqd.qk_norm_rope(q, k, p, f, q_weight=Tensor((64,), torch.bfloat16)),
                 lambda: aqd.qk_norm_rope(q, k, p, f, q_weight=w, k_weight=Tensor((128,), torch.float32)), lambda: aqd.qk_norm_rope(q, k, p, f, q_out=heads(n=5)),
                 lambda: aqd.qk_norm_rope(q, k, p, f, cache=c, slots=slots), lambda: aqd.qk_norm_rope(q, k, p, f, cache=c, v=k),
                 lambda: aqd.qk_norm_rope(q, k, p, f, cache=a_cache(1), v=k, slots=slots), lambda: aqd.qk_norm_rope(q, k, p, f, cache=c, v=heads(h=3), slots=slots),
                 lambda: aqd.qk_norm_rope(heads(strides=(2048, 256, 2)), k, p, f), lambda: aqd.qk_norm_rope(Tensor((4, 128), torch.bfloat16), k, p, f),
                 lambda: aqd.cache_write(c, q, q, slots), lambda: aqd.cache_write(c, k, heads(h=2, dtype=torch.float16), slots), lambda: aqd.cache_write(c, k, k, ints(5)),
                 lambda: aqd.cache_read(c, ints(4, torch.int32)), lambda: aqd.cache_read(c, slots, dtype=torch.int8),
                 lambda: aqd.cache_attention(heads(d=64), c, table(), ints(4, torch.int32)), lambda: aqd.cache_attention(q, c, table(), ints(4)),
                 lambda: aqd.cache_attention(q, c, table(), ints(5, torch.int32)), lambda: aqd.cache_attention(q, c, table(), ints(4, torch.int32), starts=ints(4, torch.int32)),
                 lambda: aqd.cache_attention(q, c, Tensor((4, 8), torch.int64), ints(4, torch.int32)), lambda: aqd.cache_attention(q, c, table(), ints(4, torch.int32), out=heads(n=3)),
                 lambda: aqd.cache_attention(q, c, table(), ints(4, torch.int32), workspace=Tensor((1 << 20,), torch.uint8, None)),
                 lambda: aqd.cache_attention(q, c, table(), ints(4, torch.int32), lse=Tensor((4, 8), torch.float64)),
                 lambda: aqd.prompt_attention(q, k, heads(h=4), ints(3, torch.int32)), lambda: aqd.prompt_attention(q, heads(n=5, h=2), heads(n=5, h=2), ints(3, torch.int32)),
                 lambda: aqd.prompt_attention(q, k, k, ints(3)), lambda: aqd.prompt_attention(q, k, k, ints(3, torch.int32), kv_starts=ints(4, torch.int32)),
                 lambda: aqd.prompt_attention(q, heads(h=2, d=64), heads(h=2, d=64), ints(3, torch.int32)), lambda: aqd.prompt_attention(q, k, k, ints(0, torch.int32))):
        with pytest.raises(ValueError):
            call()
    assert [n for n in made if not n.endswith("_bytes")] == []
