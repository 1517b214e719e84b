"""Forms of the operators that are chosen by size and that smaller tests do not reach, under the bounds of tests/test_gpu_rotate.py,
test_gpu_attend.py and test_gpu_groups.py."""
import pytest
import torch

from tests import test_gpu_attend as A
from tests import test_gpu_groups as G
from tests import test_gpu_rotate as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def oqm():
    from paper_2510_18269_amd import oqm as m      # raises if the library is not built
    assert torch.cuda.is_available()
    return m


# Over 1024 waves of strips, so that a wave walks its strip on its own, batch after batch, without a barrier; pieces of 16, 2, 4 and 8 bytes.
@pytest.mark.parametrize("shape", [dict(L=28, heads=4, d=128, G=64, gs=64), dict(L=28, heads=1, d=8, G=1201, gs=8, bits=2, meta="bf16"),
                                   dict(L=28, heads=1, d=8, G=2402, gs=8, bits=2, meta="bf16"), dict(L=28, heads=1, d=8, G=4804, gs=8, bits=2)])
@pytest.mark.parametrize("T,n", [(12, 9), (20, 17), (60, 59), (120, 101), (120, 8)])
def test_keep_in_strips_of_a_wave(oqm, shape, T, n):
    G.test_keep(oqm, shape, T, n)


def test_keep_the_front_and_the_end(oqm):
    """Groups that stay where they are, and ones that all come from the end."""
    for first, n in ((0, 40), (7, 33), (40, 40)):
        mem = G.memory(oqm, n, 80, 81, L=28, heads=4, d=128, G=64, gs=64)
        try:
            before = [x.clone() for x in G.planes(mem)]
            idx = torch.arange(first, first + n, dtype=torch.int32, device="cuda")
            oqm.tom_oqm_keep_groups(mem.handle, idx, n)
            torch.cuda.synchronize()
            for x, y in zip(G.planes(mem), before):
                assert torch.equal(x[:, :n], y[:, first:first + n]) and torch.equal(x[:, n:], y[:, n:])
        finally:
            mem.close()


# Past the caches (256 MB read and written), four heads a lane: parts of 14 + 3 + 3 heads hold queries, keys and values.
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("dtype,T,in_place,norm", [("bf16", 27000, False, True), ("bf16", 27000, True, False), ("f16", 27000, True, True), ("f32", 13500, False, False)])
def test_rotate_past_the_caches(oqm, dtype, T, layout, in_place, norm):
    R.check(oqm, dtype, 128, 96, layout, T, 14, 3, norm, True, first=5000, in_place=in_place)


# One, two and four heads a lane, one after the other: 14 + 3 + 3 heads, in heads wider than a wave (their norms' sums cross waves) and not.
@pytest.mark.parametrize("d,n,dtype,T", [(2048, 2048, "bf16", 100), (2048, 2048, "bf16", 300), (2048, 1024, "bf16", 600), (2046, 1026, "f16", 120), (1024, 1024, "f32", 230),
                                         (128, 128, "bf16", 4000), (128, 128, "bf16", 8000), (80, 64, "f32", 5000)])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("layout", [0, 1])
def test_rotate_heads_of_a_lane(oqm, d, n, dtype, T, norm, layout):
    R.check(oqm, dtype, d, n, layout, T, 14, 3, norm, True)


# Along the tokens outside the folded form: every width that the channels are padded to.
@pytest.mark.parametrize("d,dtype", [(d, t) for d in (8, 40, 80, 96, 136, 192, 248) for t in ("f32", "bf16", "f16")] + [(64, "f32"), (128, "f32"), (256, "f32")])
@pytest.mark.parametrize("t_q,bits,meta", [(1, 4, "f32"), (20, 2, "bf16")])
def test_attend_along_the_tokens(oqm, d, dtype, t_q, bits, meta):
    A.check(oqm, A.Case(d=d, gs=8, axis=1, dtype=dtype, t_q=t_q, bits=bits, meta=meta, recent=t_q + 20, T=12, k=10, holes=2, seed=d))


# Few query rows: every compiled folded form.
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bits", [4, 2])
@pytest.mark.parametrize("d,gs,axis", [(64, 32, 0), (64, 64, 0), (128, 32, 0), (128, 64, 0), (128, 128, 0), (256, 32, 0), (256, 64, 0), (256, 128, 0), (64, 64, 1), (128, 64, 1), (256, 64, 1)])
def test_attend_of_one_token(oqm, d, gs, axis, bits, dtype):
    A.check(oqm, A.Case(d=d, gs=gs, axis=axis, bits=bits, dtype=dtype, T=40, k=37, holes=3, meta="bf16" if gs == 64 else "f32", seed=d + gs))


# The parts of a call are joined in one order, so that it gives the same bits every time.
@pytest.mark.parametrize("kw", [dict(), dict(t_q=50, recent=60), dict(axis=1), dict(axis=1, t_q=50, dtype="f16"), dict(dtype="f32"), dict(d=80, gs=16, t_q=9),
                                dict(gs=16, t_q=100, recent=100), dict(d=256, gs=32, t_q=3), dict(G=196, T=300, k=300, every=True, heads=1)])
def test_attend_repeats_itself(oqm, kw):
    c = A.Case(**{**dict(T=60, k=50), **kw})
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    t = A.H.DT[c.dtype]
    codes, meta, _ = A.stored(c, g)
    Hq = c.heads * c.repeat
    h = oqm.tom_oqm_create(oqm.make_config(c.layers, c.heads, Hq, c.d, c.G, c.gs, c.T, qaxis=c.axis, in_dtype=t[0], out_dtype=t[0]))
    try:
        oqm.tom_oqm_bind(h, codes, meta, torch.empty(16, device="cuda"))
        oqm.tom_oqm_set_num_groups(h, c.T)
        q = torch.randn((Hq, c.t_q, c.d), generator=g, device="cuda").to(t[1])
        rows = [torch.randn((c.heads, n, c.d), generator=g, device="cuda").to(t[1]) for n in (c.front, c.front, c.recent, c.recent)]
        size = oqm.tom_oqm_attend_workspace_bytes(h, c.t_q, c.front + c.k * c.G + c.recent)
        got = []
        for i in range(6):
            out, lse = torch.empty_like(q), torch.empty((Hq, c.t_q), device="cuda")
            ws = torch.empty(size, dtype=torch.uint8, device="cuda").random_(0, 255)
            oqm.tom_oqm_attend(h, 0, q, out, None, c.k, *rows, lse=lse, workspace=ws)
            got.append((out, lse))
        torch.cuda.synchronize()
        assert all(torch.equal(out, got[0][0]) and torch.equal(lse, got[0][1]) for out, lse in got)
    finally:
        oqm.tom_oqm_destroy(h)
