"""How many rows a sequence has after some of a draft were kept (`tom_oqm_keep_rows`), where its rows or counts are at the ends of their ranges."""
import pytest
import torch

from tests.paged import Batch
from tests.test_gpu_pages import oqm  # noqa: F401

pytestmark = pytest.mark.gpu

TOP = 2 ** 31 - 1


@pytest.mark.parametrize("in_place", [False, True])
def test_rows_behind_the_table_are_counted(oqm, in_place):  # noqa: F811
    b = Batch(rows=[10, 3, 20, 7, 0, 5], new=[4, 1, 2, 3, 1, 2])
    pages, width = b.pages(oqm), 5
    capacity = b.width * b.page_rows
    rows = [10, capacity, capacity + 5, TOP, -7, TOP - 2]
    counts = [2, 1, 2, 5, 1, 2]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    pages.rows.copy_(ints(rows))
    before = pages.k.clone(), pages.v.clone()
    out = pages.rows if in_place else torch.full((b.B,), -3, dtype=torch.int32, device="cuda")
    # every index is the place that the row has: nothing moves
    oqm.tom_oqm_keep_rows(pages, ints([list(range(width))] * b.B), ints(counts), out)
    assert out.tolist() == [min(max(r, 0) + c, TOP) for r, c in zip(rows, counts)]
    if not in_place:
        assert pages.rows.tolist() == rows
    for x, y in zip((pages.k, pages.v), before):
        assert torch.equal(x.nan_to_num(nan=123.0), y.nan_to_num(nan=123.0))
    # counts of nothing, and a list of no columns, leave the number as it is
    pages.rows.copy_(ints(rows))
    oqm.tom_oqm_keep_rows(pages, ints([[]] * b.B).reshape(b.B, 0), ints(counts), out)
    assert out.tolist() == [max(r, 0) for r in rows]
