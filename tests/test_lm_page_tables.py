"""How a page table's rows may lie: what reaches the library, and what is refused, on the CPU."""
import pytest
import torch

from paper_2007_06919_gb300 import aqd
from test_lm_attention_abi import A, a_cache, attn, cache, heads, ints, lib  # noqa: F401
from test_lm_host_checks import Tensor, made  # noqa: F401


def stride_of_a_row(monkeypatch, shape, strides):
    """ld_table as the library gets it."""
    seen = []

    class Library:
        def aqd_cache_attention(self, args, *_):
            seen.append(aqd._CACHE_ATTENTION.unpack(args))
            return 0

        def __getattr__(self, name):
            return lambda *_: 1 << 20

    monkeypatch.setattr(aqd, "_calls", Library)
    table = Tensor(shape, torch.int32, 0, strides)
    aqd.cache_attention(heads(n=shape[0]), a_cache(), table, ints(shape[0], torch.int32), workspace=Tensor((1 << 20,), torch.uint8, 0))
    return seen[0][-2]


@pytest.mark.parametrize("shape,strides,want", [((4, 8), (8, 1), 8), ((4, 8), (20, 1), 20), ((4, 8), (0, 1), 0), ((4, 1), (0, 0), 0), ((4, 1), (3, 7), 3)])
def test_rows_apart_and_one_row_for_all(made, monkeypatch, shape, strides, want):  # noqa: F811
    assert stride_of_a_row(monkeypatch, shape, strides) == want


@pytest.mark.parametrize("strides", [(0, 1), (3, 1), (8, 1), (1, 1)])
def test_a_single_row_of_any_stride(made, monkeypatch, strides):  # noqa: F811
    ld = stride_of_a_row(monkeypatch, (1, 8), strides)
    assert ld == 0 or ld >= 8


@pytest.mark.parametrize("strides", [(1, 1), (7, 1), (8, 2), (0, 2)])
def test_rows_that_overlap_in_part(made, strides):  # noqa: F811
    with pytest.raises(ValueError, match="page_table"):
        aqd.cache_attention(heads(), a_cache(), Tensor((4, 8), torch.int32, 0, strides), ints(4, torch.int32))
    assert [n for n in made if not n.endswith("_bytes")] == []


def test_the_entry_point_takes_one_row_for_all(lib):  # noqa: F811
    def why(**more):
        # (a lengths pointer of 0 is refused after the table's stride is looked at: nothing is launched)
        assert lib.aqd_cache_attention(attn(lens=0, **more), cache(), A, 1 << 30, None) == 1
        return aqd.load().aqd_last_error().decode()

    assert "lengths" in why(lt=0) and "lengths" in why(lt=8) and "lengths" in why(lt=0, cols=0)
    for lt in (-1, 1, 7):
        assert "ld_table" in why(lt=lt)
