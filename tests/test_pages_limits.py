"""How much of a kind the calls on pages take, as the header counts it (no GPU is touched: every call here is refused)."""
import math

import pytest
import torch

from tests.test_operator_refusals import Fake, refuses
from tests.test_pages_refusals import I32, keeps, oqm, pages  # noqa: F401


def tensor(shape, dtype):
    """What Pages.create asks of a dense tensor on a device."""
    class T(Fake):
        device = "cuda:0"
        def dim(self): return len(self.shape)
        def stride(self, i=None): return self.strides if i is None else self.strides[i]
        def numel(self): return math.prod(self.shape)
    t = T(shape, dtype)
    t.strides = tuple(math.prod(shape[i + 1:]) for i in range(len(shape)))
    return t


@pytest.mark.parametrize("dtype,channels,heads", [("f32", 256, 32), ("f32", 8, 1024), ("bf16", 256, 64), ("f16", 8, 2048)])
def test_columns_of_kept_rows_go_by_the_element_size(oqm, dtype, channels, heads):  # noqa: F811
    """2^12 columns of 16 bytes a row, in 2^20 sequences: a lane more than a launch has.  In float32 that is half as many channels as in 16 bits."""
    n, e = 2 ** 20, 4 if dtype == "f32" else 2
    assert heads * 2 * channels * e // 16 == 2 ** 12
    p = pages(oqm, dtype={"f32": oqm.TOM_F32, "bf16": oqm.TOM_BF16, "f16": oqm.TOM_F16}[dtype], channels=channels, heads=heads, n_layers=1, n_pages=2, page_rows=1,
              row_stride=channels, head_stride=channels, page_stride=heads * channels, layer_stride=2 * heads * channels, sequences=n, table_pages=1)
    refuses(oqm, "lanes", keeps(oqm, p), oqm.TOM_ERR_UNSUPPORTED)


def test_columns_of_a_row(oqm):  # noqa: F811
    """2^31 of them, of one sequence."""
    heads, layers = 2 ** 14, 2 ** 12
    p = pages(oqm, dtype=oqm.TOM_F32, channels=64, heads=heads, n_layers=layers, n_pages=1, page_rows=1, row_stride=64, head_stride=64, page_stride=heads * 64,
              layer_stride=heads * 64, sequences=1, table_pages=1)
    refuses(oqm, "pieces", keeps(oqm, p, Fake((1, 3), I32), Fake((1,), I32), Fake((1,), I32)), oqm.TOM_ERR_UNSUPPORTED)


@pytest.mark.parametrize("shape", [(1, 2 ** 32 + 5, 1, 1, 8), (2 ** 31, 1, 1, 1, 8), (1, 1, 2 ** 32 + 1, 1, 8), (1, 1, 1, 2 ** 33, 8)])
def test_pools_of_more_than_a_size_holds(oqm, shape):  # noqa: F811
    """Sizes are 32 bits in the pages: a larger one is refused, not cut to its low bits."""
    with pytest.raises(AssertionError, match="2\\^31"):
        oqm.Pages.create(tensor(shape, torch.bfloat16), tensor(shape, torch.bfloat16), tensor((4, 5), I32), tensor((4,), I32), tensor((5,), I32))


def test_tables_of_more_than_a_size_holds(oqm):  # noqa: F811
    pool = (1, 20, 2, 16, 64)
    for table, rows in (((1, 2 ** 32 + 5), (1,)), ((2 ** 32 + 4, 1), (2 ** 32 + 4,))):
        with pytest.raises(AssertionError, match="2\\^31"):
            oqm.Pages.create(tensor(pool, torch.bfloat16), tensor(pool, torch.bfloat16), tensor(table, I32), tensor(rows, I32))


def test_lists_of_more_than_a_size_holds(oqm):  # noqa: F811
    n = 2 ** 32 + 3
    mask = Fake((3, 1), torch.int64)
    for parents, starts in ((Fake((n,), I32), Fake((2,), I32)), (Fake((3,), I32), Fake((n,), I32)), (Fake((n,), I32), None)):
        with pytest.raises(AssertionError, match="2\\^31"):
            oqm.tom_oqm_draft_tree(parents, starts, mask)
    with pytest.raises(AssertionError, match="2\\^31"):
        oqm.tom_oqm_keep_rows(pages(oqm, sequences=1), Fake((1, n), I32), Fake((1,), I32), Fake((1,), I32))
