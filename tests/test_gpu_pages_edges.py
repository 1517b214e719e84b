"""Attention over pages at the borders of its rules and with what its header allows and no ordinary call does, against its definition in float64.  How far
it may be off is derived in `paged.Batch.attention`."""
import math
import random

import pytest
import torch

from tests import paged
from tests import test_gpu_pages as pages_tests
from tests.paged import Batch
from tests.test_gpu_pages import oqm  # noqa: F401

pytestmark = pytest.mark.gpu


def two_parts(b):
    """Whether the header promises probabilities in two 16-bit parts: up to 16 query rows of a KV head on average, not rounded."""
    return b.T * b.repeat <= 16 * b.B


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("repeat,extra", [(9, 1), (9, 37), (15, 3), (16, 0), (1, 720), (7, 61)])
def test_two_parts_up_to_the_average_that_the_header_names(oqm, dtype, repeat, extra):  # noqa: F811
    """48 sequences with a token each, and some tokens more anywhere in the batch."""
    new = [1 + extra // 48 + (1 if i < extra % 48 else 0) for i in range(48)]
    b = Batch(dtype=dtype, rows=[(13 * i) % 90 for i in range(48)], new=new, heads=1, repeat=repeat, d=64, layers=1, layer=0)
    assert two_parts(b)
    got = pages_tests.call(oqm, b, b.pages(oqm))
    pages_tests.close(b, got, b.attention(None, True, b.d ** -0.5, 0.0, None, one_part=False))


# ---- numbers on the device that make no sense ------------------------------------------------------------------------


# (heads, repeat, rows, new, one each): every way of cutting, and every way to find a block (of one sequence, of up to 64, of more, of more than are looked
# through, by position)
CUTS = {
    **{name: form + (False,) for name, form in pages_tests.FORMS.items()},
    "one": (1, 3, [700], [9], False),
    "parts of more than 64": (1, 2, [(i * 29) % 400 for i in range(90)], [1 + i % 2 for i in range(90)], False),
    "blocks of more than 64": (8, 3, [(13 * i) % 97 for i in range(80)], [30 + i % 7 for i in range(80)], False),
    "blocks of more than 512": (8, 2, [(i * i * 7) % 61 for i in range(600)], [(i % 3) for i in range(600)], False),
    "one each": (2, 3, [(i * 29) % 400 for i in range(20)], [1] * 20, True),
    "one each, no parts": (8, 2, [(i * 7) % 61 for i in range(600)], [1] * 600, True),
}


def wrong_starts(b):
    B, T = b.B, b.T
    rng = random.Random(B)
    yield [0] + [9999999] * B
    yield [T] * (B + 1)
    yield [T if i % 2 else 0 for i in range(B + 1)]
    yield [0 if i % 2 else T for i in range(B + 1)]
    yield [-5] + [T - i for i in range(B)]
    yield [rng.randint(-2 ** 31, 2 ** 31 - 1) for _ in range(B + 1)]
    yield [rng.randint(0, T) for _ in range(B + 1)]


class Margins:
    """A tensor in the middle of a larger one that holds a pattern."""

    def __init__(self, shape, dtype, fill):
        n = math.prod(shape)
        self.whole = torch.full((n + 2 * 4096,), 55, dtype=dtype, device="cuda")
        self.inner = self.whole[4096:4096 + n].view(shape)
        self.inner.fill_(fill)

    def untouched(self):
        return bool((self.whole[:4096] == 55).all() and (self.whole[-4096:] == 55).all())


@pytest.mark.parametrize("cut", CUTS)
def test_numbers_that_make_no_sense_touch_nothing_else(oqm, cut):  # noqa: F811
    heads, repeat, rows, new, one_each = CUTS[cut]
    b = Batch(d=64, heads=heads, repeat=repeat, rows=rows, new=new, layers=1, layer=0, one_each=one_each)
    pages, T, Hq = b.pages(oqm), b.T, heads * repeat
    q, size = b.q.cuda(), oqm.tom_oqm_attend_pages_workspace_bytes(pages, T, Hq)
    mask = torch.full((T, 1), 0x5555, dtype=torch.int64, device="cuda")
    good = pages.rows.clone(), pages.table.clone(), None if one_each else pages.starts.clone()
    pools = pages.k.clone(), pages.v.clone()

    def wrong():
        if not one_each:
            for starts in wrong_starts(b):
                yield starts, None, None
        yield None, [(-7, 2 ** 31 - 1, 0, -2 ** 31, b.width * b.page_rows)[i % 5] for i in range(b.B)], None
        yield None, None, (-2 ** 31, 2 ** 31 - 1, b.n_pages, -1)
        if not one_each:
            yield [T if i % 2 else 0 for i in range(b.B + 1)], [2 ** 31 - 1] * b.B, (b.n_pages, 0)

    for starts, counts, entries in wrong():
        for t, x in zip((pages.rows, pages.table, pages.starts), good):
            if x is not None:
                t.copy_(x)
        if starts is not None:
            pages.starts.copy_(torch.tensor([max(-2 ** 31, min(2 ** 31 - 1, x)) for x in starts], dtype=torch.int32))
        if counts is not None:
            pages.rows.copy_(torch.tensor(counts, dtype=torch.int32))
        if entries is not None:
            pages.table.view(-1)[::2] = torch.tensor([entries[i % len(entries)] for i in range((pages.table.numel() + 1) // 2)], dtype=torch.int32, device="cuda")
        given = [t.clone() for t in (pages.rows, pages.table, q, mask)]
        # whose each token is by starts that are cut to the call's tokens
        at = [min(max(x, 0), T) for x in (list(range(T + 1)) if one_each else pages.starts.tolist())]
        somebodys = torch.zeros(T, dtype=torch.bool)
        for first, behind in zip(at, at[1:]):
            somebodys[first:behind] = True
        for fill in (-1, 3, 0):            # what an earlier call may have left in the workspace
            out, lse, ws = Margins((Hq, T, 64), torch.bfloat16, 7.0), Margins((Hq, T), torch.float32, 7.0), Margins((size,), torch.uint8, 0)
            ws.inner.view(torch.int32).fill_(fill)
            for m in (None, mask):
                oqm.tom_oqm_attend_pages(pages, 0, q, out.inner, mask=m, lse=lse.inner, workspace=ws.inner)
            torch.cuda.synchronize()
            assert out.untouched() and lse.untouched() and ws.untouched()
            assert (out.inner[:, ~somebodys] == 7.0).all() and (lse.inner[:, ~somebodys] == 7.0).all()
            for t, x in zip((pages.rows, pages.table, q, mask), given):
                assert torch.equal(t, x)
            for t, x in zip((pages.k, pages.v), pools):
                assert torch.equal(t.view(torch.int16), x.view(torch.int16))
    # and what makes sense again is right
    for t, x in zip((pages.rows, pages.table, pages.starts), good):
        if x is not None:
            t.copy_(x)
    pages_tests.close(b, pages_tests.call(oqm, b, pages), b.attention(None, True, b.d ** -0.5, 0.0, None, not two_parts(b)))


# ---- rows that a token does not see ----------------------------------------------------------------------------------


def not_finite(b, s, row, value):
    """The key and value of a row become `value` in every third channel, in the pool alone."""
    P = b.page_rows
    for x in (b.k, b.v):
        x[:, b.table_list[s][row // P], :, row % P, ::3] = value


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new", [[3, 1], [9, 2], [40, 9], [180, 3]])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("softcap,scale", [(0.0, None), (0.5, None), (20.0, None), (100.0, 0.02), (500.0, 2.0)])
def test_what_is_not_seen_may_hold_anything_under_a_cap(oqm, dtype, new, value, softcap, scale):  # noqa: F811
    """Token 1 of the first sequence is seen by itself alone and holds what is not finite; then, without a mask, the last tokens do, which those in front of
    them do not see.  Scores near zero, near the cap and above it: the ways to take a tanh are chosen by the scores' size, of unseen ones too."""
    b = Batch(dtype=dtype, d=64, heads=1, repeat=7, rows=[20, 40], new=new, layers=1, layer=0)
    masks = [[i for i in range(j + 1) if i != 1 or j == 1] for n in new for j in range(n)]
    used = 64 ** -0.5 if scale is None else scale
    words = max(1, (max(new) + 63) // 64)
    for bits, keep, row in ((masks, [j != 1 for j in range(b.T)], b.rows[0] + 1), (None, [j != new[0] - 1 for j in range(b.T)], b.rows[0] + new[0] - 1)):
        want = b.attention(bits, True, used, softcap, None, dtype != "f32" and not two_parts(b))
        k, v = b.k.clone(), b.v.clone()
        not_finite(b, 0, row, value)
        out, lse = pages_tests.call(oqm, b, b.pages(oqm), None if bits is None else paged.to_words(bits, words), softcap=softcap, scale=scale)
        b.k, b.v = k, v
        keep = torch.tensor(keep)
        assert torch.isfinite(out[:, keep]).all() and torch.isfinite(lse[:, keep]).all()
        assert ((out.double() - want[0]).abs() / want[2])[:, keep].max() <= 1
        assert ((lse.double() - want[1]).abs() / want[3])[:, keep].max() <= 1


# ---- batches whose sequences are not alike ---------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("repeat,rows,new", [
    (2, [0] + [(37 * i) % 700 for i in range(63)], [300] + [1] * 63),           # a prompt among single tokens, by the few form
    (7, [30] + [(37 * i) % 700 for i in range(20)], [600] + [1] * 20),          # by blocks of many rows
    (7, [2500] + [40] * 9, [1] + [130] * 9)])                                   # a single token with many rows among prompts
def test_prompts_beside_single_tokens(oqm, dtype, repeat, rows, new):  # noqa: F811
    b = Batch(dtype=dtype, d=64, heads=1, repeat=repeat, rows=rows, new=new, layers=1, layer=0, page_rows=50)
    pages_tests.close(b, pages_tests.call(oqm, b, b.pages(oqm)), b.attention(None, True, 0.125, 0.0, None, dtype != "f32" and not two_parts(b)))


@pytest.mark.parametrize("one_each", [False, True])
def test_a_long_sequence_that_is_not_cut(oqm, one_each):  # noqa: F811
    """So many sequences that none is cut, and one of them with many rows."""
    b = Batch(rows=[20000 if i == 411 else (i * 7) % 40 for i in range(800)], new=[1] * 800, heads=4, repeat=1, d=64, layers=1, layer=0, page_rows=64, one_each=one_each)
    pages = b.pages(oqm)
    assert oqm.tom_oqm_attend_pages_workspace_bytes(pages, 800, 4) == 0
    pages_tests.close(b, pages_tests.call(oqm, b, pages), b.attention(None, True, 0.125, 0.0))


@pytest.mark.parametrize("dtype,d", [("bf16", 256), ("f16", 256), ("bf16", 200), ("f16", 72)])
@pytest.mark.parametrize("sequences", [40, 70])
@pytest.mark.parametrize("causal", [True, False])
def test_blocks_in_the_order_of_what_they_see(oqm, dtype, d, sequences, causal):  # noqa: F811
    """More blocks than run at a time and no parts, in 16 bits of each width; among up to 64 sequences and among more."""
    b = Batch(dtype=dtype, d=d, heads=8, repeat=3, rows=[(29 * i) % 180 for i in range(sequences)], new=[22 + i % 9 for i in range(sequences)], layers=1, layer=0)
    pages = b.pages(oqm)
    assert oqm.tom_oqm_attend_pages_workspace_bytes(pages, b.T, 24) == 0 and not two_parts(b)
    pages_tests.close(b, pages_tests.call(oqm, b, pages, causal=causal), b.attention(None, causal, d ** -0.5, 0.0, None, True))


# ---- the same call again ---------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("cut", CUTS)
def test_every_cut_repeats_itself_bit_for_bit(oqm, cut, dtype):  # noqa: F811
    heads, repeat, rows, new, one_each = CUTS[cut]
    b = Batch(dtype=dtype, d=128, heads=heads, repeat=repeat, rows=rows, new=new, layers=1, layer=0, one_each=one_each)
    pages = b.pages(oqm)
    g = torch.Generator().manual_seed(5)
    prior = torch.randn(b.q.shape, generator=g).to(paged.DTYPE[dtype]), torch.randn(b.q.shape[:2], generator=g)
    first = pages_tests.call(oqm, b, pages, prior=prior, softcap=3.0)
    assert torch.isfinite(first[0]).all()
    for _ in range(5):
        again = pages_tests.call(oqm, b, pages, prior=prior, softcap=3.0)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# ---- products that pass float32's range, and tables of no pages ------------------------------------------------------


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cut", ["a few", "up to 64", "halved tiles", "prompts", "one each"])
def test_a_token_whose_products_pass_the_range_leaves_the_others_alone(oqm, cut, dtype):  # noqa: F811
    """The first token of each sequence has queries of 1e37: scores pass float32's range, or come near it, and there is no prior."""
    heads, repeat, rows, new, one_each = CUTS[cut]
    b = Batch(dtype=dtype, d=64, heads=heads, repeat=repeat, rows=rows, new=new, layers=1, layer=0, one_each=one_each)
    for s in range(0, b.B, 2 if one_each else 1):
        if new[s] > (0 if one_each else 1):
            b.q[:, b.starts_list[s]] = 1e37 * torch.sign(b.q[:, b.starts_list[s]].float()).to(b.q.dtype)
    keep = b.q.float().abs().amax((0, 2)) < 1e30
    assert 0 < keep.sum() < b.T
    for scale, softcap in ((0.125, 0.0), (10.0, 0.0), (0.125, 20.0)):
        out, lse = pages_tests.call(oqm, b, b.pages(oqm), scale=scale, softcap=softcap)
        b.q, q = torch.where(keep[None, :, None], b.q, 0.0), b.q
        want = b.attention(None, True, scale, softcap, None, dtype != "f32" and not two_parts(b))
        b.q = q
        assert ((out.double() - want[0]).abs() / want[2])[:, keep].max() <= 1
        seen = keep[None] & (want[1] > -math.inf)
        assert ((lse.double() - want[1]).abs() / want[3])[seen].max() <= 1


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("cut", ["a few", "up to 64", "halved tiles", "many blocks", "prompts", "one each"])
def test_tables_of_no_pages(oqm, cut, dtype):  # noqa: F811
    """No row has a place: nothing but a prior is seen, nothing is written to the pool, and queries are turned all the same."""
    heads, repeat, rows, new, one_each = CUTS[cut]
    b = Batch(dtype=dtype, d=64, heads=heads, repeat=repeat, rows=rows, new=new, layers=1, layer=0, one_each=one_each)
    full = b.pages(oqm)
    pages = oqm.Pages.create(full.k, full.v, torch.empty((b.B, 0), dtype=torch.int32, device="cuda"), full.rows, full.starts)
    out, lse = pages_tests.call(oqm, b, pages)
    assert (out == 0).all() and (lse == -math.inf).all()
    g = torch.Generator().manual_seed(1)
    prior = torch.randn(b.q.shape, generator=g).to(paged.DTYPE[dtype]), torch.randn(b.q.shape[:2], generator=g)
    out, lse = pages_tests.call(oqm, b, pages, prior=prior)
    assert torch.equal(out, prior[0])
    assert ((lse - prior[1]).abs() <= 2.0 ** -20 * (1 + prior[1].abs())).all()
    before = pages.k.clone(), pages.v.clone()
    x = torch.randn((b.T, heads * (repeat + 2), 64), device="cuda").to(paged.DTYPE[dtype])
    q_out = torch.zeros((b.T, heads * repeat, 64), dtype=x.dtype, device="cuda")
    oqm.tom_oqm_append_rows(pages, 0, oqm.Rotary.create(64), torch.zeros(b.T, dtype=torch.int64, device="cuda"), x[:, heads * repeat:heads * (repeat + 1)],
                            x[:, heads * (repeat + 1):], q=x[:, :heads * repeat], q_out=q_out)
    assert torch.equal(q_out, x[:, :heads * repeat])
    kept = torch.full((b.B,), -3, dtype=torch.int32, device="cuda")
    oqm.tom_oqm_keep_rows(pages, torch.ones((b.B, 2), dtype=torch.int32, device="cuda"), torch.ones(b.B, dtype=torch.int32, device="cuda"), kept)
    assert kept.tolist() == [r + 1 for r in rows]
    for t, y in zip((pages.k, pages.v), before):
        assert torch.equal(t.nan_to_num(5.0), y.nan_to_num(5.0))
