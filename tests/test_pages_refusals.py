"""What the calls on pages refuse on the host, before anything is launched, and what they take without work (no GPU is touched)."""
import ctypes as C
import math

import pytest
import torch

from tests.test_operator_refusals import Fake, refuses


@pytest.fixture()
def oqm():
    from paper_2510_18269_amd import oqm as m
    return m


BF, I32, I64, F32 = torch.bfloat16, torch.int32, torch.int64, torch.float32


def config(oqm, **kw):
    """3 layers, 20 pages of 16 rows of 2 heads of 64 channels, 4 sequences of up to 50 pages, starts given."""
    v = dict(k=0x100000, v=0x200000, layer_stride=20 * 2 * 16 * 64, page_stride=2 * 16 * 64, head_stride=16 * 64, row_stride=64, n_layers=3, n_pages=20, heads=2,
             page_rows=16, channels=64, dtype=oqm.TOM_BF16, table=0x300000, rows=0x310000, starts=0x320000, sequences=4, table_pages=50)
    v.update(kw)
    return oqm.tom_oqm_pages_t(*(v[n] for n, _ in oqm.tom_oqm_pages_t._fields_))


def pages(oqm, **kw):
    return oqm.Pages(config(oqm, **kw), None, None, None, None, None)


BAD = [
    ("channels", dict(channels=0)), ("channels", dict(channels=4)), ("channels", dict(channels=100)), ("channels", dict(channels=264)),
    ("dtype", dict(dtype=3)), ("dtype", dict(dtype=-1)), ("a layer", dict(n_layers=0)), ("a layer", dict(n_pages=0)), ("a layer", dict(heads=0)),
    ("a layer", dict(page_rows=0)), ("negative", dict(sequences=-1)), ("negative", dict(table_pages=-1)), ("strides", dict(row_stride=-64)),
    ("strides", dict(layer_stride=2 ** 41)), ("multiples of 16", dict(row_stride=65)), ("multiples of 16", dict(page_stride=2 * 16 * 64 + 4)),
    ("overlap", dict(row_stride=56)), ("overlap", dict(head_stride=0)), ("overlap", dict(page_stride=16 * 64)), ("overlap", dict(layer_stride=0)),
    ("no data", dict(k=0)), ("no data", dict(v=0)), ("16-byte aligned", dict(k=0x100008)), ("table and rows", dict(table=0)), ("table and rows", dict(rows=0)),
    ("4-byte aligned", dict(table=0x300002)), ("4-byte aligned", dict(rows=0x300001)), ("4-byte aligned", dict(starts=0x300002))]
UNSUPPORTED = [("sequences", dict(sequences=2 ** 20 + 1)), ("rows per sequence", dict(table_pages=2 ** 27)),
               ("2\\^36", dict(n_pages=2 ** 25, layer_stride=2 ** 37, n_layers=1))]


def attends(oqm, p, heads=6, tokens=7, d=64, ws=1 << 30, **kw):
    shape = (heads, tokens, d)
    args = dict(q=Fake(shape), out=Fake(shape, address=0x900000), workspace=Fake((ws,), torch.uint8, address=0x40000000), layer=0)
    args.update(kw)
    return lambda: oqm.tom_oqm_attend_pages(p, args.pop("layer"), args.pop("q"), args.pop("out"), **args)


def appends(oqm, p, tokens=7, d=64, rotary_dim=64, **kw):
    turns = Fake((rotary_dim // 2,), torch.float64)
    rotary = oqm.Rotary(oqm.tom_oqm_rotary_t(rotary_dim, 0, 0, 1, 10000.0, 1.0), turns, 1.0)
    args = dict(positions=Fake((tokens,), I64), k=Fake((tokens, 2, d)), v=Fake((tokens, 2, d)), q=Fake((tokens, 6, d)), q_out=Fake((tokens, 6, d)), layer=0)
    args.update(kw)
    return lambda: oqm.tom_oqm_append_rows(p, args.pop("layer"), args.pop("rotary", rotary), args.pop("positions"), args.pop("k"), args.pop("v"), **args)


def keeps(oqm, p, idx=None, counts=None, rows_out=None):
    n = max(p.config.sequences, 0)
    return lambda: oqm.tom_oqm_keep_rows(p, idx or Fake((n, 3), I32), counts or Fake((n,), I32), rows_out or Fake((n,), I32))


@pytest.mark.parametrize("match,kw", BAD)
def test_bad_pages(oqm, match, kw):
    for call in (attends, appends, keeps):
        refuses(oqm, match, call(oqm, pages(oqm, **kw)))
    assert oqm.tom_oqm_attend_pages_workspace_bytes(pages(oqm, **kw), 7, 6) == 0


@pytest.mark.parametrize("match,kw", UNSUPPORTED)
def test_pages_that_are_not_covered(oqm, match, kw):
    for call in (attends, appends, keeps):
        refuses(oqm, match, call(oqm, pages(oqm, **kw)), oqm.TOM_ERR_UNSUPPORTED)


def test_null_pages(oqm):
    assert oqm.lib.tom_oqm_keep_rows(None, 0, 0, 0, 0, None) == oqm.TOM_ERR_INVALID_ARG
    assert oqm.lib.tom_oqm_attend_pages_workspace_bytes(None, 1, 1) == 0


@pytest.mark.parametrize("match,kw", [
    ("layer", dict(layer=3)), ("layer", dict(layer=-1)), ("q and out", dict(out=None)), ("multiple", dict(heads=5)), ("multiple", dict(heads=0)),
    ("another dtype", dict(q=Fake((6, 7, 64), F32))), ("another dtype", dict(out=Fake((6, 7, 64), torch.float16))), ("wanted", dict(d=128)), ("wanted", dict(out=Fake((6, 8, 64)))),
    ("multiples of 16", dict(q=Fake((6, 7, 64), address=0x10008))), ("multiples of 16", dict(q=Fake((6, 7, 64), strides=(7 * 68, 68, 1)))),
    ("overlap", dict(out=Fake((6, 7, 64), strides=(0, 64, 1)))), ("both", dict(prior_out=Fake((6, 7, 64)))), ("both", dict(prior_lse=Fake((6, 7), F32))),
    ("wanted", dict(prior_out=Fake((6, 6, 64)), prior_lse=Fake((6, 7), F32))), ("wanted", dict(prior_out=Fake((6, 7, 64)), prior_lse=Fake((7, 6), F32))),
    ("wanted", dict(lse=Fake((6, 8), F32))), ("overlap", dict(lse=Fake((6, 7), F32, strides=(0, 1)))), ("words", dict(mask=Fake((7, 0), I64))),
    ("8-byte", dict(mask=Fake((7, 1), I64, address=0x10004))), ("scale must be a number", dict(scale=math.nan)), ("scale must be a number", dict(scale=math.inf)),
    ("softcap", dict(softcap=-1.0)), ("softcap", dict(softcap=math.inf)), ("2\\^50", dict(scale=2.0 ** 51)), ("2\\^50", dict(scale=2.0 ** 30, softcap=2.0 ** -25)),
    ("workspace of", dict(ws=16)), ("workspace of", dict(workspace=None)), ("workspace must be", dict(workspace=Fake((1 << 30,), torch.uint8, address=0x40000008))),
    ("has no data", dict(q=Fake((6, 7, 64), address=0))), ("has no data", dict(lse=Fake((6, 7), F32, address=0)))])
def test_bad_attentions(oqm, match, kw):
    refuses(oqm, match, attends(oqm, pages(oqm), **kw))


@pytest.mark.parametrize("match,kw", [
    ("mask", dict(mask=Fake((6, 1), I64))), ("mask", dict(mask=Fake((7,), I64))), ("mask", dict(mask=Fake((7, 1), I32))), ("mask", dict(mask=Fake((7, 2), I64, strides=(1, 7)))),
    ("lse", dict(lse=Fake((6, 7), BF))), ("lse", dict(lse=Fake((42,), F32))), ("device tensor", dict(lse=5)), ("device tensor", dict(mask=0x10000)),
    ("three dimensions", dict(q=Fake((6, 7)))), ("contiguous channel", dict(q=Fake((6, 7, 64), strides=(64 * 7, 1, 7)))), ("device tensor", dict(q=Fake((6, 7, 64), is_cuda=False)))])
def test_tensors_that_are_not_what_the_call_takes(oqm, match, kw):
    with pytest.raises(AssertionError, match=match):
        attends(oqm, pages(oqm), **kw)()


def test_attentions_that_are_not_covered(oqm):
    many = (1 << 20) + 1
    refuses(oqm, "new tokens", attends(oqm, pages(oqm), tokens=many), oqm.TOM_ERR_UNSUPPORTED)
    refuses(oqm, "2\\^30", attends(oqm, pages(oqm), heads=2048, tokens=1 << 20), oqm.TOM_ERR_UNSUPPORTED)
    assert oqm.tom_oqm_attend_pages_workspace_bytes(pages(oqm), many, 6) == 0
    assert oqm.tom_oqm_attend_pages_workspace_bytes(pages(oqm), 1 << 20, 2048) == 0


def test_without_starts_there_is_one_token_each(oqm):
    p = pages(oqm, starts=None)
    refuses(oqm, "without starts", attends(oqm, p))
    refuses(oqm, "without starts", appends(oqm, p))
    assert oqm.tom_oqm_attend_pages_workspace_bytes(p, 7, 6) == 0 and oqm.tom_oqm_attend_pages_workspace_bytes(p, 4, 6) >= 0
    refuses(oqm, "without starts", lambda: oqm._check(oqm.lib.tom_oqm_draft_tree(0x1000, None, 3, 4, 0x2000, 1, None, None, None)))


def test_workspaces_go_by_sizes(oqm):
    for heads in (2, 6, 14, 64):
        for tokens in (1, 2, 5, 16, 17, 40, 100, 500, 5000):
            n = oqm.tom_oqm_attend_pages_workspace_bytes(pages(oqm, table_pages=4000), tokens, heads)
            assert n % 16 == 0 and n == oqm.tom_oqm_attend_pages_workspace_bytes(pages(oqm, table_pages=5000), tokens, heads)
            assert n > 0 or tokens * heads > 1000
    assert oqm.tom_oqm_attend_pages_workspace_bytes(pages(oqm), 0, 6) == 0
    assert oqm.tom_oqm_attend_pages_workspace_bytes(pages(oqm), 7, 5) == 0
    assert oqm.tom_oqm_attend_pages_workspace_bytes(pages(oqm, table_pages=1), 7, 6) == 0   # nothing to be cut


@pytest.mark.parametrize("match,kw", [
    ("layer", dict(layer=3)), ("k and v", dict(k=None)), ("k and v", dict(v=None)), ("both", dict(q_out=None)), ("both", dict(q=None)),
    ("given for q", dict(q=None, q_out=None, q_norm=Fake((0,), F32))), ("dtype and channels", dict(k=Fake((7, 2, 64), torch.float16))),
    ("dtype and channels", dict(v=Fake((6, 2, 64)))), ("dtype and channels", dict(q=Fake((7, 6, 128)), q_out=Fake((7, 6, 128)))),
    ("heads", dict(k=Fake((7, 3, 64)))), ("heads", dict(q_out=Fake((7, 5, 64)))), ("overlap", dict(q_out=Fake((7, 6, 64), strides=(64, 64, 1)))),
    ("rotary_dim", dict(rotary_dim=66)), ("norm_eps", dict(norm_eps=-1.0)), ("norm_eps", dict(norm_eps=math.nan)), ("positions", dict(positions=None)),
    ("8-byte", dict(positions=Fake((7,), I64, address=0x10004))), ("aligned to their elements", dict(k=Fake((7, 2, 64), address=0x10001)))])
def test_bad_appends(oqm, match, kw):
    refuses(oqm, match, appends(oqm, pages(oqm), **kw))


def test_appends_that_are_not_covered(oqm):
    n = 1 << 30
    refuses(oqm, "2\\^31", appends(oqm, pages(oqm), tokens=n), oqm.TOM_ERR_UNSUPPORTED)


def test_bad_keeps(oqm):
    p = pages(oqm)
    refuses(oqm, "must be non-NULL", lambda: oqm._check(oqm.lib.tom_oqm_keep_rows(C.byref(p.config), None, 3, 0x1000, 0x2000, None)))
    refuses(oqm, "must be non-NULL", lambda: oqm._check(oqm.lib.tom_oqm_keep_rows(C.byref(p.config), 0x1000, 3, None, 0x2000, None)))
    refuses(oqm, "must be non-NULL", lambda: oqm._check(oqm.lib.tom_oqm_keep_rows(C.byref(p.config), 0x1000, 3, 0x1000, None, None)))
    refuses(oqm, "width", lambda: oqm._check(oqm.lib.tom_oqm_keep_rows(C.byref(p.config), 0x1000, -1, 0x1000, 0x2000, None)))
    refuses(oqm, "4-byte", lambda: oqm._check(oqm.lib.tom_oqm_keep_rows(C.byref(p.config), 0x1002, 3, 0x1000, 0x2000, None)))
    refuses(oqm, "lanes", keeps(oqm, pages(oqm, sequences=2 ** 20, n_layers=1, heads=512, layer_stride=0, page_stride=512 * 16 * 64), Fake((2 ** 20, 3), I32),
                                Fake((2 ** 20,), I32), Fake((2 ** 20,), I32)), oqm.TOM_ERR_UNSUPPORTED)
    for bad in (dict(idx=Fake((4, 3), I64)), dict(counts=Fake((3,), I32)), dict(rows_out=Fake((4,), I64)), dict(idx=Fake((4, 3), I32, strides=(1, 4)))):
        with pytest.raises(AssertionError):
            keeps(oqm, p, **bad)()


@pytest.mark.parametrize("match,args", [
    ("negative", (0x1000, 0x2000, -1, 4, 0x3000, 1, None, None)), ("negative", (0x1000, 0x2000, 1, -4, 0x3000, 1, None, None)),
    ("words", (0x1000, 0x2000, 1, 4, 0x3000, 0, None, None)), ("words", (0x1000, 0x2000, 1, 4, 0x3000, 65, None, None)),
    ("non-NULL", (None, 0x2000, 1, 4, 0x3000, 1, None, None)), ("non-NULL", (0x1000, 0x2000, 1, 4, None, 1, None, None)),
    ("4-byte", (0x1002, 0x2000, 1, 4, 0x3000, 1, None, None)), ("4-byte", (0x1000, 0x2001, 1, 4, 0x3000, 1, None, None)),
    ("8-byte", (0x1000, 0x2000, 1, 4, 0x3004, 1, None, None)), ("8-byte", (0x1000, 0x2000, 1, 4, 0x3000, 1, 0x1004, None)),
    ("8-byte", (0x1000, 0x2000, 1, 4, 0x3000, 1, None, 0x1004))])
def test_bad_trees(oqm, match, args):
    refuses(oqm, match, lambda: oqm._check(oqm.lib.tom_oqm_draft_tree(*args, None)))


def test_trees_that_are_not_covered(oqm):
    for args in ((0x1000, 0x2000, 2 ** 20 + 1, 4, 0x3000, 1), (0x1000, 0x2000, 1, 2 ** 24 + 1, 0x3000, 1)):
        refuses(oqm, "at most", lambda: oqm._check(oqm.lib.tom_oqm_draft_tree(*args, None, None, None)), oqm.TOM_ERR_UNSUPPORTED)


def test_no_work_is_no_error(oqm):
    p = pages(oqm, sequences=0)
    attends(oqm, p, tokens=0, ws=0)()
    attends(oqm, p, tokens=3, ws=0)()          # nobody's tokens
    appends(oqm, p, tokens=0)()
    appends(oqm, p, tokens=3)()
    keeps(oqm, p, Fake((0, 3), I32), Fake((0,), I32), Fake((0,), I32))()
    attends(oqm, pages(oqm), tokens=0, ws=0)()
    oqm._check(oqm.lib.tom_oqm_draft_tree(None, None, 0, 0, None, 1, None, None, None))


def test_pages_from_tensors(oqm):
    """What Pages.create asks of its tensors."""
    class T(Fake):
        def dim(self): return len(self.shape)
        def stride(self, i=None): return self.strides if i is None else self.strides[i]
        device = "cuda:0"
    def make(shape, dtype=BF, strides=None, **kw):
        f = T(shape, dtype, strides, **kw)
        n, dense = 1, []
        for s in reversed(shape):
            dense.insert(0, n)
            n *= s
        f.strides = tuple(strides or dense)
        f.numel = lambda: n
        return f
    pool = (3, 20, 2, 16, 64)
    good = dict(k=make(pool), v=make(pool, address=0x20000), table=make((4, 5), I32), rows=make((4,), I32), starts=make((5,), I32))
    p = oqm.Pages.create(**good)
    assert (p.config.n_layers, p.config.n_pages, p.config.heads, p.config.page_rows, p.config.channels) == pool
    assert (p.config.layer_stride, p.config.page_stride, p.config.head_stride, p.config.row_stride) == (40960, 2048, 1024, 64)
    assert (p.config.sequences, p.config.table_pages, p.config.dtype) == (4, 5, oqm.TOM_BF16)
    assert oqm.Pages.create(**{**good, "starts": None}).config.starts is None
    for bad in (dict(v=make((3, 20, 2, 16, 128))), dict(v=make(pool, torch.float16)), dict(k=make(pool, torch.float64), v=make(pool, torch.float64)),
                dict(v=make(pool, strides=(40960, 2048, 64, 128, 1))), dict(k=make((20, 2, 16, 64)), v=make((20, 2, 16, 64))), dict(table=make((20,), I32)),
                dict(table=make((4, 5), I64)), dict(rows=make((3,), I32)), dict(starts=make((4,), I32)), dict(rows=make((4,), I32, is_cuda=False))):
        with pytest.raises(AssertionError):
            oqm.Pages.create(**{**good, **bad})
