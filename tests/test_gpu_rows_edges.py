"""Trees, rows appended and rows kept where starts, rows, table, parents or lists make no sense: nothing but what is a sequence's is written, and what makes sense again
is right.  (tests/test_pages_lanes.py runs the same on the host under AddressSanitizer.)"""
import random

import pytest
import torch

from tests import paged
from tests.paged import Batch
from tests.test_gpu_pages import oqm  # noqa: F401
from tests.test_gpu_pages_edges import Margins, wrong_starts

pytestmark = pytest.mark.gpu

BATCHES = {"one": ([20], [13]), "some": ([70, 0, 33, 15], [5, 1, 30, 20]), "many": ([(i * 7) % 40 for i in range(90)], [(i * 5) % 4 for i in range(90)])}


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def cut(v):
    return [max(-2 ** 31, min(2 ** 31 - 1, x)) for x in v]


@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("words", [1, 3])
def test_trees(oqm, batch, words):  # noqa: F811
    new = BATCHES[batch][1]
    b = Batch(rows=[0] * len(new), new=new, heads=1, repeat=1, d=8, layers=1, layer=0)
    rng = random.Random(2)
    parents = [rng.choice([-1, -2 ** 31, 2 ** 31 - 1, rng.randint(-3, 40), max(0, j - 1)]) for n in new for j in range(n)]
    for starts in list(wrong_starts(b)) + [b.starts_list]:
        mask, positions = Margins((b.T, words), torch.int64, 7), Margins((b.T,), torch.int64, 7)
        given = ints(cut(starts))
        oqm.tom_oqm_draft_tree(ints(parents), given, mask.inner, positions.inner)
        torch.cuda.synchronize()
        assert mask.untouched() and positions.untouched() and given.tolist() == cut(starts)
        at = [min(max(x, 0), b.T) for x in starts]
        nobodys = torch.ones(b.T, dtype=torch.bool)
        for first, behind in zip(at, at[1:]):
            nobodys[first:behind] = False
        assert (mask.inner[nobodys] == 7).all() and (positions.inner[nobodys] == 7).all()
    want = paged.ancestors([p if 0 <= p < j else -1 for p, j in zip(parents, [j for n in new for j in range(n)])], new)
    assert torch.equal(mask.inner.cpu(), paged.to_words(want, words)) and positions.inner.tolist() == [len(w) - 1 for w in want]


def pool_of(oqm, b):  # noqa: F811
    """The pages with their pools between margins."""
    pages = b.pages(oqm)
    k, v = (Margins(x.shape, x.dtype, 0) for x in (pages.k, pages.v))
    for m, x in ((k, pages.k), (v, pages.v)):
        m.inner.copy_(x.nan_to_num(3.0))
    return oqm.Pages.create(k.inner, v.inner, pages.table, pages.rows, pages.starts), k, v


def in_a_table(b, table):
    """Which pages stand in the table at all."""
    there = torch.zeros(b.n_pages, dtype=torch.bool)
    for p in table.flatten().tolist():
        if 0 <= p < b.n_pages:
            there[p] = True
    return there


def variants(b, pages):
    good = pages.rows.clone(), pages.table.clone(), pages.starts.clone()

    def back():
        for t, x in zip((pages.rows, pages.table, pages.starts), good):
            t.copy_(x)

    for starts in wrong_starts(b):
        back()
        pages.starts.copy_(ints(cut(starts)))
        yield
    for rows in ([-7] * b.B, [2 ** 31 - 1] * b.B, [b.width * b.page_rows - 1] * b.B):
        back()
        pages.rows.copy_(ints(rows))
        yield
    back()
    pages.table.view(-1)[::2] = ints([(-2 ** 31, 2 ** 31 - 1, b.n_pages, -1)[i % 4] for i in range((pages.table.numel() + 1) // 2)])
    yield
    back()


@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_appends(oqm, batch, dtype):  # noqa: F811
    rows, new = BATCHES[batch]
    b = Batch(dtype=dtype, rows=rows, new=new, heads=2, repeat=2, d=64, layers=2, layer=1)
    pages, k, v = pool_of(oqm, b)
    x = torch.randn((b.T, 8, 64), device="cuda").to(paged.DTYPE[dtype])
    rotary, positions = oqm.Rotary.create(64), torch.zeros(b.T, dtype=torch.int64, device="cuda")

    def append():
        q_out = Margins((b.T, 4, 64), x.dtype, 7.0)
        oqm.tom_oqm_append_rows(pages, 1, rotary, positions, x[:, 4:6], x[:, 6:], q=x[:, :4], q_out=q_out.inner)
        torch.cuda.synchronize()
        assert q_out.untouched() and k.untouched() and v.untouched()

    for _ in variants(b, pages):
        before = k.inner.clone(), v.inner.clone()
        append()
        free = ~in_a_table(b, pages.table)
        for m, y in zip((k, v), before):
            assert torch.equal(m.inner[0], y[0]) and torch.equal(m.inner[:, free], y[:, free])
    append()
    for s in range(b.B):
        for j in range(new[s]):
            r, t = rows[s] + j, b.starts_list[s] + j
            page = b.table_list[s][r // b.page_rows]
            assert torch.equal(k.inner[1, page, :, r % b.page_rows], x[t, 4:6]) and torch.equal(v.inner[1, page, :, r % b.page_rows], x[t, 6:])


@pytest.mark.parametrize("batch", BATCHES)
@pytest.mark.parametrize("in_place", [False, True])
def test_keeps(oqm, batch, in_place):  # noqa: F811
    rows, new = BATCHES[batch]
    b = Batch(rows=rows, new=new, heads=2, repeat=1, d=72, layers=2, layer=0)
    pages, k, v = pool_of(oqm, b)
    rng = random.Random(4)
    width = 6
    counts = [min(n, 1 + rng.randint(0, width - 1)) for n in new]
    idx = [sorted(rng.sample(range(n), c)) + [-1] * (width - c) for n, c in zip(new, counts)]

    def keep(idx, counts):
        out = Margins((b.B,), torch.int32, -3)
        oqm.tom_oqm_keep_rows(pages, ints(idx), ints(counts), pages.rows if in_place else out.inner)
        torch.cuda.synchronize()
        assert out.untouched() and k.untouched() and v.untouched()
        return pages.rows.tolist() if in_place else out.inner.tolist()

    for _ in variants(b, pages):
        before = k.inner.clone(), v.inner.clone()
        had = pages.rows.tolist()
        assert keep(idx, counts) == [min(max(r, 0) + c, 2 ** 31 - 1) for r, c in zip(had, counts)]
        free = ~in_a_table(b, pages.table)
        for m, y in zip((k, v), before):
            assert torch.equal(m.inner[:, free], y[:, free])
    assert keep([[rng.randint(-2 ** 31, 2 ** 31 - 1) for _ in range(width)] for _ in new], [rng.randint(-2 ** 31, 2 ** 31 - 1) for _ in new]) is not None
    pages.rows.copy_(ints(rows))
    before = k.inner.clone(), v.inner.clone()
    assert keep(idx, counts) == [r + c for r, c in zip(rows, counts)]
    for s in range(b.B):
        for i in range(counts[s]):
            to, source = rows[s] + i, rows[s] + idx[s][i]
            a, c = b.table_list[s][to // b.page_rows], b.table_list[s][source // b.page_rows]
            for m, y in zip((k, v), before):
                assert torch.equal(m.inner[:, a, :, to % b.page_rows], y[:, c, :, source % b.page_rows])
