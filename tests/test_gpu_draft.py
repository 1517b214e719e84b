"""Trees of drafted tokens, rows appended to pages, accepted rows kept (`tom_oqm_draft_tree`, `tom_oqm_append_rows`, `tom_oqm_keep_rows`), and all of
them together with the attention over stored groups."""
import math
import random

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


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


# ---- trees -----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("new", [[1], [13], [64], [65], [3, 0, 200, 1, 64], [1, 1, 1], [700], [5000]])
@pytest.mark.parametrize("kind", ["tree", "chain", "roots"])
def test_trees(oqm, new, kind):
    T, words = sum(new), min(64, (max(new) + 63) // 64)
    if kind == "tree":
        parents = paged.tree(new, 5)
    else:
        parents = [j - 1 if kind == "chain" else -1 for n in new for j in range(n)]
    starts = [sum(new[:i]) for i in range(len(new) + 1)]
    first = [10 ** 12 - 7 * i for i in range(len(new))]
    mask = torch.full((T + 2, words), 7, dtype=torch.int64, device="cuda")
    positions = torch.full((T + 2,), 7, dtype=torch.int64, device="cuda")
    oqm.tom_oqm_draft_tree(ints(parents + [-1, 0]), ints(starts), mask, positions, ints(first, torch.int64))
    want = paged.ancestors(parents, new)
    assert torch.equal(mask.cpu()[:T], paged.to_words(want, words))
    which = [s for s, n in enumerate(new) for _ in range(n)]
    assert positions.tolist() == [first[s] + len(w) - 1 for s, w in zip(which, want)] + [7, 7]
    assert (mask[T:] == 7).all()             # tokens behind the last sequence are nobody's
    few = torch.empty((T, 1), dtype=torch.int64, device="cuda")
    oqm.tom_oqm_draft_tree(ints(parents), ints(starts), few)
    assert torch.equal(few.cpu(), paged.to_words(want, 1))


def test_parents_that_are_none(oqm):
    parents = [0, 5, -9, 2, 2 ** 31 - 1, 4, -2 ** 31, 7, 1]
    mask, positions = torch.empty((9, 2), dtype=torch.int64, device="cuda"), torch.empty(9, dtype=torch.int64, device="cuda")
    oqm.tom_oqm_draft_tree(ints(parents), ints([0, 9]), mask, positions)
    want = paged.ancestors([-1, -1, -1, 2, -1, 4, -1, -1, 1], [9])
    assert torch.equal(mask.cpu(), paged.to_words(want, 2)) and positions.tolist() == [len(w) - 1 for w in want]


def test_tokens_behind_the_most_that_a_draft_may_have(oqm):
    T = 65536 + 70
    mask, positions = torch.full((T + 5, 2), 7, dtype=torch.int64, device="cuda"), torch.full((T + 5,), 7, dtype=torch.int64, device="cuda")
    oqm.tom_oqm_draft_tree(ints([-1] * (T + 5)), ints([0, T, T + 5]), mask, positions)
    assert (positions[:65536] == 0).all() and (positions[65536:T] == 7).all() and (positions[T:] == 0).all()
    want = torch.zeros((65536, 2), dtype=torch.int64)
    for i in range(128):
        want[i, i // 64] = -2 ** 63 if i % 64 == 63 else 1 << (i % 64)
    assert torch.equal(mask[:65536].cpu(), want) and (mask[65536:T] == 7).all()
    assert mask[T:, 0].tolist() == [1 << i for i in range(5)] and (mask[T:, 1] == 0).all()


def test_one_token_each(oqm):
    mask, positions = torch.empty((70, 1), dtype=torch.int64, device="cuda"), torch.empty(70, dtype=torch.int64, device="cuda")
    oqm.tom_oqm_draft_tree(ints([-1] * 70), None, mask, positions, ints(list(range(70)), torch.int64))
    assert (mask == 1).all() and positions.tolist() == list(range(70))


# ---- appended rows ---------------------------------------------------------------------------------------------------


def turned(x, weight, positions, n, layout, base):
    """x [T][heads][d] in float64."""
    d = x.shape[-1]
    if weight is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight
    angle = positions.double()[:, None, None] * base ** (-torch.arange(0, n, 2, dtype=torch.float64) / n)
    one = torch.arange(n // 2) if layout == 0 else torch.arange(0, n, 2)
    two = one + (n // 2 if layout == 0 else 1)
    y = x.clone()
    y[..., one] = x[..., one] * torch.cos(angle) - x[..., two] * torch.sin(angle)
    y[..., two] = x[..., two] * torch.cos(angle) + x[..., one] * torch.sin(angle)
    assert y.shape[-1] == d
    return y


def append(oqm, b, rotary_dim, layout, norm, with_q=True, offset=0, in_place=False, positions=None):
    """Calls it on rows of one projection and checks every element of the pools and of q_out."""
    t, P = DTYPE[b.dtype], b.page_rows
    g = torch.Generator().manual_seed(b.seed + 100)
    Hq, H, base = b.heads * b.repeat, b.heads, 10000.0
    wide = torch.randn((b.T, (Hq + 2 * H) * b.d + offset), generator=g).to(t).cuda()
    x = wide[:, offset:].unflatten(1, (Hq + 2 * H, b.d))
    q, k, v = x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
    given = x.cpu().double()
    weights = [(1 + 0.2 * torch.randn(b.d, generator=g)).to(t) if norm else None for _ in range(2)]
    pages = b.pages(oqm)
    before = pages.k.cpu(), pages.v.cpu()
    if positions is None:
        positions = torch.randint(0, 100000, (b.T,), generator=g)
    q_out = q if in_place else torch.full((b.T, Hq, b.d), 7.0, dtype=t, device="cuda")
    rotary = oqm.Rotary.create(rotary_dim, layout=layout, base=base)
    dev = [None if w is None else w.cuda() for w in weights]
    oqm.tom_oqm_append_rows(pages, b.layer, rotary, positions.cuda(), k, v, q=q if with_q else None, q_out=q_out if with_q else None,
                            q_norm=dev[0] if with_q else None, k_norm=dev[1])
    torch.cuda.synchronize()
    used = b.starts_list[-1]
    # products and sums of a handful of float32 roundings, and the rounding of the type; a norm's sum of d squares adds d * 2^-24 / 2
    half, rest = torch.finfo(t).eps / 2, 2.0 ** -20 + (b.d * 2.0 ** -24 if norm else 0)

    def near(got, want):
        size = want.abs() + want.abs().amax(-1, keepdim=True)    # a turn adds two products: off by a part of the larger channel
        assert (got.double() - want).abs().sub(half * want.abs() + rest * size + torch.finfo(t).tiny).max() <= 0

    if with_q:
        near(q_out.cpu()[:used], turned(given[:, :Hq], None if weights[0] is None else weights[0].double(), positions, rotary_dim, layout, base)[:used])
        assert torch.equal(q_out.cpu()[used:], wide.cpu()[used:, offset:].unflatten(1, (Hq + 2 * H, b.d))[:, :Hq] if in_place else torch.full_like(q_out.cpu()[used:], 7.0))
    keys = turned(given[:, Hq:Hq + H], None if weights[1] is None else weights[1].double(), positions, rotary_dim, layout, base)
    got = pages.k.cpu(), pages.v.cpu()
    for s in range(b.B):
        for j in range(b.new[s]):
            row, token = b.rows[s] + j, b.starts_list[s] + j
            page = b.table_list[s][row // P] if row // P < b.width else -1
            if not 0 <= page < b.n_pages:
                continue
            near(got[0][b.layer, page, :, row % P], keys[token])
            assert torch.equal(got[1][b.layer, page, :, row % P].double(), given[token, Hq + H:])
            for x, y in zip(got, before):
                x[b.layer, page, :, row % P] = y[b.layer, page, :, row % P]
    for x, y in zip(got, before):            # nothing else has been written
        assert torch.equal(x.nan_to_num(nan=123.0), y.nan_to_num(nan=123.0))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("norm", [False, True])
def test_appends(oqm, dtype, layout, norm):
    append(oqm, Batch(dtype=dtype, rows=[70, 0, 33, 15], new=[5, 1, 3, 20]), 128, layout, norm)


@pytest.mark.parametrize("d,rotary_dim", [(8, 2), (64, 64), (72, 30), (80, 80), (96, 48), (128, 64), (256, 256), (256, 6)])
@pytest.mark.parametrize("layout", [0, 1])
def test_appends_of_other_sizes(oqm, d, rotary_dim, layout):
    append(oqm, Batch(d=d, rows=[70, 0], new=[5, 1], page_rows=7), rotary_dim, layout, True)


@pytest.mark.parametrize("order", ["lphrc", "plhrc", "lprhc", "hlprc"])
def test_appends_to_other_orders(oqm, order):
    append(oqm, Batch(order=order, rows=[3, 90], new=[30, 1], page_rows=50, layers=3), 128, 0, False)


@pytest.mark.parametrize("offset", [1, 2, 4, 8])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 256)])
def test_appends_from_odd_addresses(oqm, offset, dtype, d):
    append(oqm, Batch(dtype=dtype, d=d, rows=[3, 90], new=[3, 1]), d, 0, True, offset=offset)


def test_appends_in_place_without_queries_and_one_each(oqm):
    append(oqm, Batch(), 128, 0, True, in_place=True)
    append(oqm, Batch(behind=3), 128, 0, True, in_place=True)
    append(oqm, Batch(behind=3), 64, 1, False)
    append(oqm, Batch(), 128, 0, True, with_q=False)
    append(oqm, Batch(rows=[0, 15, 16, 17], new=[1] * 4, one_each=True), 128, 1, False)
    append(oqm, Batch(rows=[5], new=[1], one_each=True), 128, 0, True)


def test_appends_to_pages_that_are_not_there(oqm):
    append(oqm, Batch(rows=[14, 30, 3], new=[20, 4, 2], holes=[(0, 1), (2, 0)]), 128, 0, False)
    b = Batch(rows=[14, 30], new=[40, 4])
    b.table_list, b.width = [t[:2] for t in b.table_list], 2
    append(oqm, b, 128, 0, True)


def test_appends_of_many_tokens_and_sequences(oqm):
    append(oqm, Batch(rows=[i % 40 for i in range(300)], new=[(i * 7) % 5 for i in range(300)], d=64, heads=1, repeat=2, layers=1, layer=0), 64, 0, False)
    append(oqm, Batch(rows=[100, 7], new=[3000, 1], d=64, heads=1, repeat=3, layers=1, layer=0, page_rows=64), 64, 1, True)


def test_far_positions(oqm):
    append(oqm, Batch(), 128, 0, False, positions=torch.arange(9) + 10 ** 6)


# ---- kept rows -------------------------------------------------------------------------------------------------------


def keep(oqm, b, idx, counts, width, in_place=False):
    pages = b.pages(oqm)
    want, P = [pages.k.cpu(), pages.v.cpu()], b.page_rows
    for s in range(b.B):
        for x in want:
            old = x.clone()
            for i in range(min(max(counts[s], 0), width)):
                j = idx[s][i]
                to, source = b.rows[s] + i, b.rows[s] + j
                if not i <= j < b.new[s] or to // P >= b.width or source // P >= b.width:
                    continue
                a, c = b.table_list[s][to // P], b.table_list[s][source // P]
                if 0 <= a < b.n_pages and 0 <= c < b.n_pages:
                    x[:, a, :, to % P] = old[:, c, :, source % P]
    rows = pages.rows if in_place else torch.full((b.B,), -3, dtype=torch.int32, device="cuda")
    oqm.tom_oqm_keep_rows(pages, ints(idx).reshape(b.B, width), ints(counts), rows)
    torch.cuda.synchronize()
    assert rows.tolist() == [r + min(max(c, 0), width) for r, c in zip(b.rows, counts)]
    for x, y in zip((pages.k.cpu(), pages.v.cpu()), want):
        assert torch.equal(x.nan_to_num(nan=123.0), y.nan_to_num(nan=123.0))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [8, 72, 128, 256])
@pytest.mark.parametrize("in_place", [False, True])
def test_keeps(oqm, dtype, d, in_place):
    b = Batch(dtype=dtype, d=d, rows=[70, 0, 33, 15], new=[5, 1, 30, 20], layers=3)
    keep(oqm, b, [[0, 2, 4] + [0] * 9, [0] * 12, list(range(3, 27, 2)), [1] + [0] * 11], [3, 1, 12, 0], 12, in_place)


@pytest.mark.parametrize("order", ["lphrc", "plhrc", "lprhc", "hlprc"])
def test_keeps_in_other_orders(oqm, order):
    keep(oqm, Batch(order=order, rows=[3, 90], new=[30, 9], page_rows=7), [[9, 10, 11, 20, 29], [0, 1, 2, 3, 8]], [5, 5], 5)


def test_keeps_of_indices_and_counts_that_are_wrong(oqm):
    b = Batch(rows=[70, 0, 33], new=[5, 1, 9])
    keep(oqm, b, [[0, 5, 2 ** 31 - 1], [-1, 0, 0], [-2 ** 31, 4, 8]], [3, 2 ** 31 - 1, 3], 3)
    keep(oqm, b, [[0, 1, 2], [0, 0, 0], [0, 1, 2]], [-4, 0, 3], 3)
    keep(oqm, b, [[], [], []], [1, 2, 3], 0)


def test_keeps_on_pages_that_are_not_there(oqm):
    keep(oqm, Batch(rows=[14, 30, 3], new=[40, 4, 2], holes=[(0, 1), (2, 0)]), [[1, 2, 20, 39], [1, 2, 3, 0], [1, 0, 0, 0]], [4, 3, 1], 4)
    b = Batch(rows=[14, 30], new=[40, 4])
    b.table_list, b.width = [t[:2] for t in b.table_list], 2
    keep(oqm, b, [[1, 17, 18, 39], [0, 1, 2, 3]], [4, 4], 4)


def test_keeps_of_many(oqm):
    rng = random.Random(3)
    new = [rng.randint(0, 40) for _ in range(200)]
    counts = [rng.randint(0, n) for n in new]
    idx = [sorted(rng.sample(range(n), c)) + [0] * (40 - c) for n, c in zip(new, counts)]
    keep(oqm, Batch(rows=[rng.randint(0, 50) for _ in new], new=new, d=64, heads=1), idx, counts, 40)
    keep(oqm, Batch(rows=[0], new=[500], d=64, heads=1), [list(range(7, 500, 3))], [165], 165, True)


# ---- together --------------------------------------------------------------------------------------------------------


def test_a_step_of_drafts_over_stored_frames(oqm):
    """Two conversations: frames in a memory of each, system rows in front, answers so far in pages, a draft's tree.  Rows are appended, the groups
    attended to, the pages joined, the accepted path kept and a next token decoded, against one softmax in float64 over all that a token sees."""
    L, H, R, d, G, k = 2, 2, 3, 64, 16, 5
    Hq, t, base = H * R, torch.bfloat16, 10000.0
    g = torch.Generator().manual_seed(11)
    rand = lambda *n: torch.randn(n, generator=g).to(t)  # noqa: E731
    memories, frames = [], []
    for s in range(2):
        mem = oqm.Memory.allocate(oqm.make_config(L, H, Hq, d, G, 32, 8))
        kv = rand(6, L, H, G, d).cuda(), rand(6, L, H, G, d).cuda()
        oqm.tom_oqm_quantize_append(mem.handle, 0, L, 6, *kv)
        active = [torch.empty((L, H, 6 * G, d), dtype=t, device="cuda") for _ in range(2)]
        oqm.tom_oqm_dequant_gather(mem.handle, 0, L, ints([list(range(6))] * L), 6, 6, *active)
        memories.append(mem)
        frames.append([x.cpu().double() for x in active])
    chosen = [[0, 2, 3, 4, 5], [1, 2, 3, 4, 5]]
    front = rand(L, H, 4, d), rand(L, H, 4, d)
    P, n_pages = 8, 16
    pool = [torch.full((L, n_pages, H, P, d), math.nan, dtype=t, device="cuda") for _ in range(2)]
    table = [[3, 7, 1, 12], [9, 0, 4, 5]]
    rows_had = [13, 2]
    told = [[rand(L, H, r, d), rand(L, H, r, d)] for r in rows_had]
    for s in range(2):
        for i in range(rows_had[s]):
            for x, y in zip(pool, told[s]):
                x[:, table[s][i // P], :, i % P] = y[:, :, i].cuda()
    rows = ints(rows_had)
    new = [7, 4]
    T, starts = 11, ints([0, 7, 11])
    parents = [-1, 0, 0, 1, 1, 3, 2] + [-1, 0, 1, 0]
    pages = oqm.Pages.create(*pool, ints(table), rows, starts)
    rotary = oqm.Rotary.create(d, base=base)
    mask, positions = torch.empty((T, 1), dtype=torch.int64, device="cuda"), torch.empty(T, dtype=torch.int64, device="cuda")
    oqm.tom_oqm_draft_tree(ints(parents), starts, mask, positions, ints([1000, 2000], torch.int64))
    seen = paged.ancestors(parents, new)
    at = [0, 7]

    def layer_step(pages, layer, x, positions, mask, sizes, begins):
        """Queries turned, rows appended, and the answer over groups and pages, as a model's layer asks for it."""
        q_out = torch.empty((x.shape[0], Hq, d), dtype=t, device="cuda")
        oqm.tom_oqm_append_rows(pages, layer, rotary, positions, x[:, Hq:Hq + H], x[:, Hq + H:], q=x[:, :Hq], q_out=q_out)
        n = x.shape[0]
        q, out = q_out.transpose(0, 1), torch.empty((n, Hq, d), dtype=t, device="cuda").transpose(0, 1)
        lse = torch.empty((Hq, n), device="cuda")
        for s in range(2):
            m = oqm.tom_oqm_attend_workspace_bytes(memories[s].handle, sizes[s], 4 + k * G)
            part = torch.empty((Hq, sizes[s]), device="cuda")
            cut = slice(begins[s], begins[s] + sizes[s])
            oqm.tom_oqm_attend(memories[s].handle, layer, q[:, cut], out[:, cut], idx=ints(chosen[s]), k_eff=k, front_k=front[0][layer].cuda(),
                               front_v=front[1][layer].cuda(), lse=part, workspace=torch.empty(m, dtype=torch.uint8, device="cuda"))
            lse[:, cut] = part
        ws = torch.empty(oqm.tom_oqm_attend_pages_workspace_bytes(pages, n, Hq), dtype=torch.uint8, device="cuda")
        oqm.tom_oqm_attend_pages(pages, layer, q, out, mask=mask, prior_out=out, prior_lse=lse, lse=lse, workspace=ws)
        return q_out.cpu().double(), out.cpu().double(), lse.cpu().double()

    def whole(layer, q, s, extra_k, extra_v):
        """One query of [Hq][d] over everything in one softmax."""
        res, sums = [], []
        for h in range(Hq):
            j = h // R
            group = torch.cat([torch.arange(c * G, c * G + G) for c in chosen[s]])
            kk = torch.cat([front[0][layer, j].double(), frames[s][0][layer, j][group], extra_k[:, j]])
            vv = torch.cat([front[1][layer, j].double(), frames[s][1][layer, j][group], extra_v[:, j]])
            w = kk @ q[h] / math.sqrt(d)
            sums.append(torch.logsumexp(w, 0))
            res.append(torch.softmax(w, 0) @ vv)
        return torch.stack(res), torch.stack(sums)

    def near(got, want, values):
        # the prior's output and the result are rounded to bfloat16 (2^-8 each), probabilities may be too, frames are as the gather rounds them (2^-8 of a key: a score
        # of up to 16 * 2^-8 * |q||k| / d^0.5 is seen by its parts; 2^-6 of the values' size covers the random sum of 64 such terms)
        assert (got - want).abs().max() <= 3 * 2.0 ** -8 * values.abs().max() + 2.0 ** -6

    made = {}
    for layer in range(L):
        x = rand(T, Hq + 2 * H, d).cuda()
        q, out, lse = layer_step(pages, layer, x, positions, mask, new, at)
        keys = turned(x[:, Hq:Hq + H].cpu().double(), None, positions.cpu(), d, 0, base).to(t).double()
        values = x[:, Hq + H:].cpu().double()
        made[layer] = keys, values
        for s in range(2):
            for j in range(new[s]):
                up = [at[s] + i for i in seen[at[s] + j]]
                ek = torch.cat([told[s][0][layer].transpose(0, 1).double(), keys[up]])
                ev = torch.cat([told[s][1][layer].transpose(0, 1).double(), values[up]])
                o, total = whole(layer, q[at[s] + j], s, ek, ev)
                near(out[:, at[s] + j], o, ev)
                assert (lse[:, at[s] + j] - total).abs().max() < 2.0 ** -6
    # the path 0, 1, 3, 5 of the first draft and 0, 3 of the second are accepted
    oqm.tom_oqm_keep_rows(pages, ints([[0, 1, 3, 5], [0, 3, 0, 0]]), ints([4, 2]), rows)
    assert rows.tolist() == [17, 4]
    path = [[0, 1, 3, 5], [7, 10]]
    step = oqm.Pages.create(*pool, pages.table, rows)    # one token each from here
    positions = ints([1004, 2002], torch.int64)
    for layer in range(L):
        x = rand(2, Hq + 2 * H, d).cuda()
        q, out, lse = layer_step(step, layer, x, positions, None, [1, 1], [0, 1])
        keys = turned(x[:, Hq:Hq + H].cpu().double(), None, positions.cpu(), d, 0, base).to(t).double()
        for s in range(2):
            ek = torch.cat([told[s][0][layer].transpose(0, 1).double(), made[layer][0][path[s]], keys[s:s + 1]])
            ev = torch.cat([told[s][1][layer].transpose(0, 1).double(), made[layer][1][path[s]], x[s:s + 1, Hq + H:].cpu().double()])
            o, total = whole(layer, q[s], s, ek, ev)
            near(out[:, s], o, ev)
            assert (lse[:, s] - total).abs().max() < 2.0 ** -6
    for mem in memories:
        mem.close()


@pytest.mark.parametrize("new", [[3, 1, 2], [40, 9, 30]])
def test_a_captured_step_follows_parents_starts_rows_and_tables(oqm, new):
    """Tree, rows appended, attention and kept rows as one graph, replayed for other conversations with eager work between: as the eager calls, bit for bit."""
    b = Batch(rows=[70, 0, 333], new=new, d=64, heads=2, repeat=3, page_rows=16, spare=30)
    t, T, H, Hq = DTYPE[b.dtype], b.T, 2, 6
    g = torch.Generator().manual_seed(3)
    base = b.pages(oqm)
    k0, v0, rows, starts, table = base.k.clone(), base.v.clone(), base.rows, base.starts, base.table
    k0.nan_to_num_(0.5), v0.nan_to_num_(0.5)
    x = torch.randn((T, Hq + 2 * H, 64), generator=g).to(t).cuda()
    parents, first = torch.zeros(T, dtype=torch.int32, device="cuda"), ints([100, 2000, 30], torch.int64)
    mask, positions = torch.zeros((T, 1), dtype=torch.int64, device="cuda"), torch.zeros(T, dtype=torch.int64, device="cuda")
    q_out, out, lse = torch.zeros((T, Hq, 64), dtype=t, device="cuda"), torch.zeros((T, Hq, 64), dtype=t, device="cuda"), torch.zeros((Hq, T), device="cuda")
    idx, counts = ints([[0, 2, 5], [0, 1, 2], [1, 3, 29]]), ints([2, 1, 2])
    ws = torch.empty(oqm.tom_oqm_attend_pages_workspace_bytes(base, T, Hq), dtype=torch.uint8, device="cuda")
    rotary = oqm.Rotary.create(64)

    def step():
        oqm.tom_oqm_draft_tree(parents, starts, mask, positions, first)
        for layer in range(b.layers):
            oqm.tom_oqm_append_rows(base, layer, rotary, positions, x[:, Hq:Hq + H], x[:, Hq + H:], q=x[:, :Hq], q_out=q_out)
            oqm.tom_oqm_attend_pages(base, layer, q_out.transpose(0, 1), out.transpose(0, 1), mask=mask, lse=lse, workspace=ws)
        oqm.tom_oqm_keep_rows(base, idx, counts, rows)

    def load(turn):
        base.k.copy_(k0), base.v.copy_(v0)
        shift = min(turn, 2)
        starts.copy_(torch.tensor([max(0, s - shift) for s in b.starts_list], dtype=torch.int32))
        rows.copy_(torch.tensor([max(0, r - 13 * turn) for r in b.rows], dtype=torch.int32))
        table.copy_(torch.tensor(b.table_list, dtype=torch.int32).reshape(table.shape).roll(turn % 2, 0))
        parents.copy_(torch.tensor(paged.tree(new, 5 + turn), dtype=torch.int32))
        for y in (mask, positions, q_out, out, lse):
            y.zero_()
        ws.fill_(255)

    results = lambda: [y.clone() for y in (mask, positions, q_out, out, lse, base.k, base.v, rows)]  # noqa: E731
    load(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in (0, 1, 3, 0, 2):
        load(turn)
        step()
        want = results()
        load(turn)
        graph.replay()
        torch.cuda.synchronize()
        for got, y in zip(results(), want):
            assert torch.equal(got, y)
    assert torch.isfinite(out).all() and (mask[:starts[-1]] != 0).any()
