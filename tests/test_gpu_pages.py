"""Attention over pages (`tom_oqm_attend_pages`) against its definition in float64; what is nobody's row holds NaN.  How far it may be off is
derived in `paged.Batch.attention`."""
import math

import pytest
import torch

from tests import paged
from tests.paged import DTYPE, Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def oqm():
    from paper_2510_18269_amd import oqm as m      # raises if the library is not built
    assert torch.cuda.is_available()
    return m


def one_part(b):
    """Whether probabilities may enter the products as one 16-bit part: where sequences have more than 16 query rows of a head."""
    return b.dtype != "f32" and -(-b.T // b.B) * b.repeat > 16


def call(oqm, b, pages, mask=None, causal=True, scale=None, softcap=0.0, prior=None, tokens_first=True, lse=True, **kw):
    Hq, t = b.heads * b.repeat, DTYPE[b.dtype]
    q = b.q.cuda()
    if tokens_first:
        q = q.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.full((b.T, Hq, b.d), 7.0, dtype=t, device="cuda").transpose(0, 1) if tokens_first else torch.full((Hq, b.T, b.d), 7.0, dtype=t, device="cuda")
    sums = torch.full((Hq, b.T), 7.0, device="cuda") if lse else None
    size = oqm.tom_oqm_attend_pages_workspace_bytes(pages, b.T, Hq)
    ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    p = {} if prior is None else {"prior_out": prior[0].cuda(), "prior_lse": prior[1].cuda()}
    oqm.tom_oqm_attend_pages(pages, b.layer, q, out, mask=None if mask is None else mask.cuda(), causal=causal, scale=scale, softcap=softcap, lse=sums,
                             workspace=ws, **p, **kw)
    torch.cuda.synchronize()
    return out.cpu(), sums.cpu() if lse else None


def close(b, got, want):
    out, lse, bound, lse_bound = want
    used = b.starts_list[-1]
    o = got[0].double()
    assert torch.isfinite(o).all()
    worst = float(((o - out).abs() / bound)[:, :used].max())
    assert worst <= 1
    assert (o[:, used:] == 7.0).all()      # tokens behind the last sequence are left alone
    if got[1] is not None:
        x, y = got[1].double()[:, :used], lse[:, :used]
        empty = y == -math.inf
        assert torch.equal(x == -math.inf, empty)
        worst = float(((x - y).abs() / lse_bound[:, :used])[~empty].amax()) if (~empty).any() else 0.0
        assert worst <= 1
        assert (got[1][:, used:] == 7.0).all()


def check(oqm, b, parents=None, masks=None, words=None, causal=True, softcap=0.0, scale=None, prior=None, **kw):
    if parents is not None:
        masks = paged.ancestors(parents, b.new)
    mask = None
    if masks is not None:
        mask = paged.to_words(masks + [[0]] * b.behind, words or max(1, (max(b.new) + 63) // 64))
    got = call(oqm, b, b.pages(oqm), mask, causal, scale, softcap, prior, **kw)
    p = None if prior is None else (prior[0].double(), prior[1].double())
    close(b, got, b.attention(masks, causal, b.d ** -0.5 if scale is None else scale, softcap, p, one_part(b)))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [8, 64, 72, 80, 128, 192, 256])
def test_types_and_channels(oqm, dtype, d):
    check(oqm, Batch(dtype=dtype, d=d, rows=[70, 0, 33], new=[5, 1, 3]))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows", [0, 1, 15, 16, 31, 32, 33, 63, 64, 127, 128, 129, 500])
def test_one_token_of_one_sequence(oqm, dtype, rows):
    check(oqm, Batch(dtype=dtype, rows=[rows], new=[1], one_each=True))


@pytest.mark.parametrize("repeat", [1, 2, 5, 8, 16, 17, 40])
def test_query_heads_of_a_head(oqm, repeat):
    check(oqm, Batch(repeat=repeat, heads=3, rows=[40, 7], new=[1, 1], one_each=True))
    check(oqm, Batch(repeat=repeat, heads=1, rows=[40, 7], new=[3, 2]))


@pytest.mark.parametrize("page_rows", [1, 3, 7, 16, 32, 50, 64, 100, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_page_sizes(oqm, page_rows, dtype):
    check(oqm, Batch(dtype=dtype, page_rows=page_rows, rows=[200, 31, 64, 0], new=[4, 9, 1, 2]), parents=paged.tree([4, 9, 1, 2], page_rows))


@pytest.mark.parametrize("order", ["lphrc", "plhrc", "lprhc", "hlprc", "prlhc"])
def test_orders_of_the_pool(oqm, order):
    check(oqm, Batch(order=order, rows=[90, 20], new=[3, 3], layers=3, layer=2))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new", [[1, 20, 7], [64], [65, 1], [130, 3, 64, 0, 1]])
def test_trees(oqm, dtype, new):
    rows = [(37 * i + 50) % 90 for i in range(len(new))]
    check(oqm, Batch(dtype=dtype, rows=rows, new=new, page_rows=7), parents=paged.tree(new, 3))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("rows,new", [([0], [300]), ([100, 0], [77, 150]), ([1, 40, 3], [1, 33, 200])])
def test_prompts(oqm, dtype, causal, rows, new):
    check(oqm, Batch(dtype=dtype, rows=rows, new=new, page_rows=64), causal=causal)


@pytest.mark.parametrize("new", [[2, 3], [30, 11]])
def test_masks_that_leave_rows_empty(oqm, new):
    masks = [[j for j in range(n) if (i * 5 + j * 3) % 4 == 1] for n in new for i in range(n)]  # any bits, also later tokens'
    masks[0], masks[-1] = [], []
    check(oqm, Batch(rows=[0, 0], new=new), masks=masks)
    check(oqm, Batch(rows=[0, 40], new=new), masks=masks)
    check(oqm, Batch(rows=[5, 0], new=new, dtype="f32"), masks=masks)


def test_masks_of_fewer_and_more_words_than_tokens(oqm):
    new = [100, 70]
    masks = [[j for j in range(i + 1) if j < 64] for n in new for i in range(n)]
    check(oqm, Batch(rows=[10, 90], new=new), masks=masks, words=1)
    check(oqm, Batch(rows=[10, 90], new=[3, 2]), masks=paged.ancestors([-1, 0, 0, -1, 0], [3, 2]), words=3)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("softcap", [0.5, 20.0, 100.0])
def test_caps(oqm, dtype, softcap):
    check(oqm, Batch(dtype=dtype, spread=3.0), softcap=softcap)
    check(oqm, Batch(dtype=dtype, spread=3.0, new=[30, 41, 3]), softcap=softcap)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new", [[1, 1, 1], [20, 33, 1]])
def test_a_prior_part(oqm, dtype, new):
    b = Batch(dtype=dtype, rows=[70, 0, 300], new=new)
    g = torch.Generator().manual_seed(5)
    prior = torch.randn(b.q.shape, generator=g).to(DTYPE[dtype]), torch.randn(b.q.shape[:2], generator=g) * 4
    prior[1][0, 0] = -math.inf
    prior[0][0, 0] = math.nan                # is not looked at
    prior[1][1, 0], prior[1][2, 0] = 60.0, -90.0
    check(oqm, b, parents=paged.tree(new, 2), prior=prior)
    # with masks that leave tokens without rows, and with nothing at all
    b = Batch(dtype=dtype, rows=[0, 0, 3], new=new)
    masks = [[] for _ in range(b.T)]
    check(oqm, b, masks=masks, prior=prior)


@pytest.mark.parametrize("d", [64, 80, 256])
def test_outputs_may_be_the_prior_itself(oqm, d):
    b = Batch(d=d, rows=[70, 0, 600], new=[1, 4, 2])
    g = torch.Generator().manual_seed(5)
    Hq = b.heads * b.repeat
    for order in ((0, 1), (1, 0)):
        prior = torch.randn((Hq, b.T, d), generator=g).bfloat16(), torch.randn((Hq, b.T), generator=g)
        out = prior[0].cuda().permute(*order, 2).contiguous().permute(*order, 2)
        lse = prior[1].cuda().permute(*order).contiguous().permute(*order)
        pages = b.pages(oqm)
        ws = torch.empty(oqm.tom_oqm_attend_pages_workspace_bytes(pages, b.T, Hq), dtype=torch.uint8, device="cuda")
        oqm.tom_oqm_attend_pages(pages, b.layer, b.q.cuda(), out, prior_out=out, prior_lse=lse, lse=lse, workspace=ws)
        close(b, (out.cpu(), lse.cpu()), b.attention(None, True, d ** -0.5, 0.0, (prior[0].double(), prior[1].double()), one_part(b)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page_rows,new", [(16, [2, 1, 5]), (50, [40, 1, 33]), (7, [1, 1, 1])])
def test_pages_that_are_not_there(oqm, dtype, page_rows, new):
    rows = [page_rows * 6 + 2, page_rows * 3, 5]
    holes = [(0, 0), (0, 2), (0, 3), (1, 0), (1, 1), (1, 2), (2, 0)]  # the last two sequences keep little or nothing
    check(oqm, Batch(dtype=dtype, rows=rows, new=new, page_rows=page_rows, holes=holes))


def test_rows_past_the_table_are_nobodys(oqm):
    """A table of fewer pages than the rows need: what is behind it is not there."""
    b = Batch(rows=[60, 20], new=[10, 3], page_rows=16)
    for s in range(2):
        for i in range(3, b.width):
            b.table_list[s][i] = -1
    want = b.attention(None, True, b.d ** -0.5, 0.0, None, one_part(b))
    b.table_list = [t[:3] for t in b.table_list]
    b.width = 3
    close(b, call(oqm, b, b.pages(oqm)), want)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("new", [[3, 1], [40, 9]])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_rows_that_a_token_does_not_see_may_hold_anything(oqm, dtype, new, value):
    """The first sequence's token 1 is seen by itself alone, and its key and value are not finite."""
    b = Batch(dtype=dtype, rows=[20, 40], new=new)
    masks = [[i for i in range(j + 1) if i != 1 or j == 1] for n in new for j in range(n)]
    want = b.attention(masks, True, b.d ** -0.5, 0.0, None, one_part(b))
    P, row = b.page_rows, b.rows[0] + 1
    b.k[:, b.table_list[0][row // P], :, row % P, ::3] = value
    b.v[:, b.table_list[0][row // P], :, row % P, ::3] = value
    out, lse = call(oqm, b, b.pages(oqm), paged.to_words(masks, 1))
    keep = torch.ones(b.T, dtype=torch.bool)
    keep[1] = False
    assert torch.isfinite(out[:, keep]).all()
    worst = float(((out.double() - want[0]).abs() / want[2])[:, keep].max()), float(((lse.double() - want[1]).abs() / want[3])[:, keep].max())
    assert max(worst) <= 1


@pytest.mark.parametrize("new", [[1, 1, 1, 1], [4, 40, 0, 1]])
def test_long_sequences_among_short_ones(oqm, new):
    check(oqm, Batch(rows=[9000, 3, 700, 0], new=new, heads=1, d=64, page_rows=50, layers=1, layer=0))


def test_many_sequences(oqm):
    rows = [(i * i * 7) % 61 for i in range(700)]
    check(oqm, Batch(rows=rows, new=[1] * 700, heads=1, repeat=2, d=64, layers=1, layer=0, page_rows=32, one_each=True))
    check(oqm, Batch(rows=rows, new=[(i % 4) for i in range(700)], heads=1, repeat=3, d=64, layers=1, layer=0, page_rows=32))


def test_more_workgroups_than_the_chip_without_parts(oqm):
    """So many blocks that none is cut: with a workspace of nothing."""
    b = Batch(rows=[5] * 500, new=[1] * 500, heads=8, repeat=2, d=64, layers=1, layer=0, page_rows=16, one_each=True)
    assert oqm.tom_oqm_attend_pages_workspace_bytes(b.pages(oqm), b.T, 16) == 0
    check(oqm, b)
    check(oqm, Batch(rows=[5] * 400, new=[2, 0, 1, 3] * 100, heads=8, repeat=2, d=64, layers=1, layer=0, page_rows=16))


def test_tokens_behind_the_last_sequence(oqm):
    check(oqm, Batch(behind=5))
    check(oqm, Batch(behind=3, new=[30, 1, 40]), parents=paged.tree([30, 1, 40], 1))


@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0])
def test_scales(oqm, scale):
    check(oqm, Batch(dtype="f32"), scale=scale)
    check(oqm, Batch(new=[20, 1, 9]), scale=scale)


def test_heads_first_without_lse(oqm):
    check(oqm, Batch(), tokens_first=False, lse=False)


def test_binary16_tails(oqm):
    """Many small probabilities beside a large one: below the last place of binary16 each, and a tenth of the result together."""
    b = Batch(dtype="f16", rows=[4000], new=[2], heads=1, repeat=2, d=64, layers=1, layer=0, page_rows=64)
    b.q = torch.zeros_like(b.q)
    b.q[..., 0] = 8.0
    P = b.page_rows
    for i in range(4002):
        key = torch.zeros(64, dtype=torch.float16)
        key[0] = 8.0 if i == 17 else -6.0            # scores of 8 and -6: e^-14 of the largest, 4000 of them 0.3 % of it
        b.k64[0][0, 0, i] = key.double()
        b.k[0, b.table_list[0][i // P], 0, i % P] = key
        value = torch.full((64,), 1.0 if i == 17 else 400.0, dtype=torch.float16)
        b.v64[0][0, 0, i] = value.double()
        b.v[0, b.table_list[0][i // P], 0, i % P] = value
    check(oqm, b)


def test_calls_repeat_themselves_bit_for_bit(oqm):
    b = Batch(rows=[9000, 300], new=[20, 3], heads=1, d=64, page_rows=50, layers=1, layer=0)
    pages = b.pages(oqm)
    first = call(oqm, b, pages)
    for _ in range(3):
        again = call(oqm, b, pages)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_a_captured_call_follows_rows_starts_and_table(oqm):
    """The graph is captured with one step's sizes and replayed with others, with eager work between."""
    b = Batch(rows=[3000, 10, 0], new=[3, 1, 2], layers=1, layer=0, d=64)
    c = Batch(rows=[100, 2990, 5], new=[1, 5, 0], layers=1, layer=0, d=64, seed=9)
    assert b.T == c.T
    width = max(b.width, c.width)
    Hq = b.heads * b.repeat
    n_pages = max(b.n_pages, c.n_pages)
    k, v = (torch.full((1, n_pages, b.heads, b.page_rows, b.d), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
    rows, starts = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    q, out = torch.zeros(b.q.shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(b.q.shape, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((Hq, b.T), device="cuda")
    pages = oqm.Pages.create(k, v, table, rows, starts)
    ws = torch.empty(oqm.tom_oqm_attend_pages_workspace_bytes(pages, b.T, Hq), dtype=torch.uint8, device="cuda")

    def load(x):
        for pool, source in ((k, x.k), (v, x.v)):
            pool.fill_(math.nan)
            pool[:, :x.n_pages] = source.cuda()
        table.fill_(-1)
        table[:, :x.width] = torch.tensor(x.table_list, dtype=torch.int32)
        rows.copy_(torch.tensor(x.rows, dtype=torch.int32))
        starts.copy_(torch.tensor(x.starts_list, dtype=torch.int32))
        q.copy_(x.q)
        out.fill_(7.0)
        lse.fill_(7.0)

    load(b)
    oqm.tom_oqm_attend_pages(pages, 0, q, out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        oqm.tom_oqm_attend_pages(pages, 0, q, out, lse=lse, workspace=ws)
    for x in (c, b, c, c, b):
        load(x)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        close(x, (out.cpu(), lse.cpu()), x.attention(None, True, x.d ** -0.5, 0.0, None, one_part(x)))


def test_another_stream(oqm):
    b = Batch()
    pages = b.pages(oqm)
    want = call(oqm, b, pages)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    got = call(oqm, b, pages, stream=stream)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_starts_that_are_wrong_stay_inside(oqm):
    """Numbers on the device that make no sense: nothing outside is touched, and what is not contradictory is right."""
    b = Batch(rows=[40, 10, 5], new=[2, 3, 1])
    pages = b.pages(oqm)
    for starts in ([0, 9999, 9999, 9999], [-5, 3, 2, 6], [6, 0, 6, 0], [2147483647, -2147483648, 5, 6]):
        pages.starts.copy_(torch.tensor(starts, dtype=torch.int32))
        call(oqm, b, pages)
    pages.starts.copy_(torch.tensor(b.starts_list, dtype=torch.int32))
    for rows in ([-7, 10, 5], [2147483647, 10, 5]):
        pages.rows.copy_(torch.tensor(rows, dtype=torch.int32))
        call(oqm, b, pages)
    pages.rows.copy_(torch.tensor(b.rows, dtype=torch.int32))
    close(b, call(oqm, b, pages), b.attention(None, True, b.d ** -0.5, 0.0, None, one_part(b)))


# Query rows of a KV head a sequence on average, and workgroups, that lead to each way of cutting: (heads, repeat, rows, new)
FORMS = {
    "a few": (2, 5, [70, 0, 33], [3, 1, 2]),
    "up to 64": (3, 7, [150, 0, 333], [9, 1, 7]),
    "halved tiles": (2, 7, [150, 0, 1333, 64], [40, 1, 77, 0]),
    "many blocks": (8, 3, [(13 * i) % 97 for i in range(70)], [30 + i % 7 for i in range(70)]),
    "prompts": (1, 7, [131, 0], [300, 333]),
}


@pytest.mark.parametrize("dtype,d,page_rows", [("bf16", 128, 50), ("f16", 72, 64), ("bf16", 256, 7), ("f16", 64, 196), ("bf16", 200, 64), ("f16", 128, 3)])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("kind", ["causal", "all", "bits, cap, prior"])
def test_every_cut_of_the_rows(oqm, form, kind, dtype, d, page_rows):
    heads, repeat, rows, new = FORMS[form]
    if len(rows) > 10 and d > 128:
        pytest.skip("takes the reference long, and the same kernel as halved tiles")
    b = Batch(dtype=dtype, d=d, page_rows=page_rows, heads=heads, repeat=repeat, rows=rows, new=new, layers=1, layer=0, behind=2,
              holes=[(0, 0)] + [(s, 1) for s in range(len(new)) if rows[s] + new[s] > page_rows][:1])
    if kind != "bits, cap, prior":
        return check(oqm, b, causal=kind == "causal")
    g = torch.Generator().manual_seed(5)
    prior = torch.randn(b.q.shape, generator=g).to(DTYPE[dtype]), torch.randn(b.q.shape[:2], generator=g) * 4
    masks = [[j for j in range(n) if (i * 5 + j * 3) % 4 == 1 or j == i - 1] for n in new for i in range(n)]
    check(oqm, b, masks=masks, prior=prior, softcap=2.0, scale=0.2)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("falling", [False, True])
def test_scores_that_float32_rounds(oqm, dtype, form, falling):
    """Scores of 2^27 and more, of which the largest takes all: steps of 128 where float32 has steps of 16, so that a maximum that is kept in float32 may be off by
    as much, but no probability beside the largest is above 2^-100.  What comes out is its value, off by a probability's rounding and the type's."""
    heads, repeat, rows, new = FORMS[form]
    b = Batch(dtype=dtype, d=64, heads=heads, repeat=repeat, rows=rows, new=new, layers=1, layer=0)
    b.q = torch.zeros_like(b.q)
    b.q[..., 0], b.q[..., 1] = 8192.0, 128.0
    P, want, top = b.page_rows, torch.zeros(b.q.shape, dtype=torch.float64), torch.zeros(b.q.shape[:2], dtype=torch.float64)
    for s in range(b.B):
        n = rows[s] + new[s]
        order = [(37 * i) % 211 for i in range(n)] if not falling else [max(0, 255 - i) for i in range(n)]
        for i, j in enumerate(order):
            key = torch.zeros(64)
            key[0], key[1] = 16384.0, float(j)
            b.k[0, b.table_list[s][i // P], :, i % P] = key.to(DTYPE[dtype])
        for own in range(new[s]):
            upto = order[:rows[s] + own + 1]
            best = max(range(len(upto)), key=lambda i: upto[i])
            same = [i for i in range(len(upto)) if upto[i] == upto[best]]
            token = b.starts_list[s] + own
            top[:, token] = 2.0 ** 27 + 128.0 * upto[best]
            # equal scores may be weighted differently, since they are off by as much as float32 rounds them: then nothing is asked of the value
            want[:, token] = b.v64[s][0, :, best].repeat_interleave(repeat, 0) if len(same) == 1 else math.nan
    got, lse = call(oqm, b, b.pages(oqm), scale=1.0)
    half = torch.finfo(DTYPE[dtype]).eps / 2
    assert torch.isfinite(got).all() and torch.isfinite(lse).all()
    one = ~want.isnan()
    assert ((got.double() - want).abs() - (2 * half + 2.0 ** -16) * want.abs())[one].max() <= 0
    assert ((lse.double() - top).abs() / top).max() <= 2.0 ** -21


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("form", FORMS)
def test_scales_far_from_the_cap(oqm, dtype, form):
    heads, repeat, rows, new = FORMS[form]
    b = Batch(dtype=dtype, d=64, heads=heads, repeat=repeat, rows=rows, new=new, layers=1, layer=0, spread=3000.0)
    check(oqm, b, softcap=1.0, scale=1e-6)
    b.q = torch.zeros_like(b.q)          # every score is zero, whatever the powers of scale / cap are
    for scale, cap in ((2.0 ** 40, 1.0), (2.0 ** 20, 2.0 ** -20), (1e-30, 1e-3), (1.0, 2.0 ** 39)):
        check(oqm, b, softcap=cap, scale=scale)


@pytest.mark.parametrize("form", ["up to 64", "halved tiles", "prompts"])
def test_a_captured_call_of_many_rows_follows_starts(oqm, form):
    heads, repeat, rows, new = FORMS[form]
    b = Batch(heads=heads, repeat=repeat, rows=rows, new=new, layers=1, layer=0, d=64)
    pages, Hq = b.pages(oqm), heads * repeat
    q, out, lse = b.q.cuda(), torch.zeros(b.q.shape, dtype=torch.bfloat16, device="cuda"), torch.zeros((Hq, b.T), device="cuda")
    ws = torch.empty(oqm.tom_oqm_attend_pages_workspace_bytes(pages, b.T, Hq), dtype=torch.uint8, device="cuda")
    oqm.tom_oqm_attend_pages(pages, 0, q, out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        oqm.tom_oqm_attend_pages(pages, 0, q, out, lse=lse, workspace=ws)
    want = out.clone(), lse.clone()
    # with fewer rows in front and fewer tokens the eager call says what a replay has to give, and with the first ones again the first results
    for less in (1, 0, 2, 0):
        pages.rows.copy_(torch.tensor([max(0, r - 40 * less) for r in rows], dtype=torch.int32))
        pages.starts.copy_(torch.tensor([max(0, x - less) for x in b.starts_list], dtype=torch.int32))
        out.zero_(), lse.zero_(), ws.fill_(255)
        oqm.tom_oqm_attend_pages(pages, 0, q, out, lse=lse, workspace=ws)
        eager = out.clone(), lse.clone()
        out.zero_(), lse.zero_(), ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        if less == 0:
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    close(b, (out.cpu(), lse.cpu()), b.attention(None, True, b.d ** -0.5, 0.0, None, one_part(b)))


def test_two_calls_at_once(oqm):
    """On two streams, each with a workspace of its own, on the same pages."""
    b = Batch(rows=[9000, 300], new=[20, 3], heads=2, d=64, page_rows=50, layers=1, layer=0)
    pages, Hq = b.pages(oqm), b.heads * b.repeat
    want = call(oqm, b, pages)
    q, size = b.q.cuda(), oqm.tom_oqm_attend_pages_workspace_bytes(pages, b.T, Hq)
    outs = [(torch.zeros(q.shape, dtype=q.dtype, device="cuda"), torch.zeros((Hq, b.T), device="cuda"), torch.empty(size, dtype=torch.uint8, device="cuda")) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for stream, (out, lse, ws) in zip(streams, outs):
            oqm.tom_oqm_attend_pages(pages, 0, q, out, lse=lse, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    for out, lse, _ in outs:
        assert torch.equal(out.cpu(), want[0]) and torch.equal(lse.cpu(), want[1])


def test_sequences_that_share_pages(oqm):
    """One prompt's pages in the tables of all, each with a last page of its own."""
    b = Batch(rows=[64, 64, 64], new=[3, 3, 3], page_rows=16, layers=1, layer=0)
    for s in (1, 2):
        b.table_list[s][:4] = b.table_list[0][:4]
        for mine, first in ((b.k64[s], b.k64[0]), (b.v64[s], b.v64[0])):
            mine[:, :, :64] = first[:, :, :64]
    check(oqm, b, parents=paged.tree(b.new, 3))


def test_more_sequences_than_lanes_and_more_blocks_than_fit(oqm):
    b = Batch(rows=[(i * i * 7) % 61 for i in range(1500)], new=[(i % 3) for i in range(1500)], heads=4, repeat=2, d=64, layers=1, layer=0, page_rows=32)
    assert oqm.tom_oqm_attend_pages_workspace_bytes(b.pages(oqm), b.T, 8) == 0
    check(oqm, b)


@pytest.mark.parametrize("heads,repeat,rows,new,d,page_rows,parts", [
    (32, 9, [2100 + i if i % 13 == 0 else 20 for i in range(40)], [2] * 40, 64, 32, False),
    (8, 3, [2100 + i if i % 13 == 0 else 20 for i in range(90)], [33] * 90, 64, 50, False),
    (1, 7, [30000], [1200], 72, 256, True)])
def test_parts_of_more_rows_than_are_looked_up_at_a_time(oqm, heads, repeat, rows, new, d, page_rows, parts):
    b = Batch(heads=heads, repeat=repeat, rows=rows, new=new, d=d, page_rows=page_rows, layers=1, layer=0, holes=[(0, 3), (0, 40)])
    assert (oqm.tom_oqm_attend_pages_workspace_bytes(b.pages(oqm), b.T, heads * repeat) > 0) == parts
    check(oqm, b)


@pytest.mark.parametrize("new", [[1, 2], [9, 5], [70, 3]])
def test_pools_whose_offsets_pass_32_bits(oqm, new):
    """Pages at the ends of a pool of 40 GiB (places counted in 16 bytes pass 2^31), K and V beside each other in it: the same as in a small pool, bit for bit."""
    b = Batch(rows=[200, 100], new=new, layers=1, layer=0, page_rows=64)
    want = call(oqm, b, b.pages(oqm))
    page = 2 * b.heads * b.page_rows * b.d
    n = 40 * 2 ** 30 // (2 * page)
    pool = torch.empty((n, 2, b.heads, b.page_rows, b.d), dtype=torch.bfloat16, device="cuda")
    at = [p if p % 3 == 0 else n - 1 - p for p in range(b.n_pages)]
    for p in range(b.n_pages):
        pool[at[p], 0], pool[at[p], 1] = b.k[0, p].cuda(), b.v[0, p].cuda()
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table = ints([[at[p] if 0 <= p < b.n_pages else -1 for p in t] for t in b.table_list])
    pages = oqm.Pages.create(pool[:, 0][None], pool[:, 1][None], table, ints(b.rows), ints(b.starts_list))
    got = call(oqm, b, pages)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # the last token of each sequence is kept as its first, and rows appended behind it come back as they were given
    idx, counts = ints([[x - 1] for x in new]), ints([1, 1])
    oqm.tom_oqm_keep_rows(pages, idx, counts, pages.rows)
    assert pages.rows.tolist() == [r + 1 for r in b.rows]
    for s in range(2):
        page_of = lambda r: at[b.table_list[s][r // 64]]  # noqa: E731
        for half, source in ((0, b.k64), (1, b.v64)):
            kept = pool[page_of(b.rows[s]), half, :, b.rows[s] % 64].cpu().double()
            assert torch.equal(kept, source[s][0, :, b.rows[s] + new[s] - 1])
    values = torch.randn((2, b.heads, b.d), dtype=torch.bfloat16, device="cuda")
    pages = oqm.Pages.create(pool[:, 0][None], pool[:, 1][None], table, ints(b.rows), None)
    oqm.tom_oqm_append_rows(pages, 0, oqm.Rotary.create(64), torch.zeros(2, dtype=torch.int64, device="cuda"), values, values)
    for s in range(2):
        for half in range(2):
            assert torch.equal(pool[at[b.table_list[s][b.rows[s] // 64]], half, :, b.rows[s] % 64], values[s])
