"""Rows read back from the cache to places of any address and stride, keys or values alone, through the C entry point."""
import pytest
import torch

from paper_2007_06919_gb300 import aqd

pytestmark = pytest.mark.gpu
CODES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def read(cache, slots, k, v):
    def part(t):
        return (0, 0, 0) if t is None else (t.data_ptr(), t.stride(0), t.stride(1))
    dt = CODES[(k if v is None else v).dtype]
    aqd._check(aqd._calls().aqd_cache_read(aqd._CACHE_ROWS.pack(slots.numel(), dt, *part(k), *part(v), slots.data_ptr()), cache.desc, aqd._stream()), "aqd_cache_read")


@pytest.mark.parametrize("dtype", list(CODES))
@pytest.mark.parametrize("kv,dim,tokens", [(1, 64, 1), (3, 192, 77), (8, 128, 300), (2, 256, 1000)])
def test_any_place(dtype, kv, dim, tokens):
    torch.manual_seed(dim)
    cache = aqd.KVCache(tokens // 32 + 2, 32, kv, dim)
    cache.data.fill_(0x5A)
    rows = torch.randn(2, tokens, kv, dim, device="cuda")
    slots = torch.randperm(cache.pages * 32, device="cuda")[:tokens]
    aqd.cache_write(cache, rows[0], rows[1], slots)
    slots[tokens // 2] = cache.pages * 32  # outside: zeros
    want = aqd.cache_read(cache, slots, dtype=dtype)
    assert (want[0][tokens // 2] == 0).all()
    for pad, order in ((1, "tokens"), (3, "heads"), (8, "tokens"), (8, "heads")):
        def place():
            if order == "tokens":
                whole = torch.full((tokens, kv, dim + 2 * pad), 7.0, device="cuda", dtype=dtype)
                return whole, whole[:, :, pad:pad + dim]
            whole = torch.full((kv, tokens, dim + 2 * pad), 7.0, device="cuda", dtype=dtype)
            return whole, whole[:, :, pad:pad + dim].transpose(0, 1)
        for keys, values in ((True, True), (True, False), (False, True)):
            (wk, k), (wv, v) = place(), place()
            read(cache, slots, k if keys else None, v if values else None)
            for there, whole, got, exact in ((keys, wk, k, want[0]), (values, wv, v, want[1])):
                assert torch.equal(got, exact) if there else (whole == 7).all()
                assert (whole[..., :pad] == 7).all() and (whole[..., pad + dim:] == 7).all()
