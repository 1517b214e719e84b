"""Attention over rows in front, stored groups and recent rows (`tom_oqm_attend`) against its definition in float64.

Tolerances.  A score differs by at most `off` = scale * sum_c |q_c k_c| * 2^-15: keys and probabilities enter the matrix
products as two 16-bit parts or exactly (a rest of 2^-17), and float32 sums of up to a few hundred terms add 2^-17 more; a
cap, whose slope is at most one, adds softcap * 2^-20.  A probability is then off by a factor of e^(2 off), so the output
by (2 off + 2^-14) * sum_j p_j |v_j| and half a step of its type; the logarithm of the sum by off + 2^-20 of its size."""
import math

import pytest
import torch

from tests import harness as H

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def oqm():
    from paper_2510_18269_amd import oqm as m      # raises if the library is not built
    assert torch.cuda.is_available()
    return m


class Case:
    def __init__(self, **kw):
        self.dtype, self.d, self.heads, self.repeat, self.G, self.gs = "bf16", 128, 2, 7, 50, 64
        self.axis, self.bits, self.meta, self.T, self.k, self.every, self.holes = 0, 4, "f32", 9, 5, False, 0
        self.t_q, self.front, self.recent, self.causal, self.softcap, self.layers = 1, 14, 33, True, 0.0, 2
        self.seed, self.spread = 1, 1.0
        for name, value in kw.items():
            assert hasattr(self, name), name
            setattr(self, name, value)


def stored(c, g):
    """Random codes and pairs, as the arrays of a memory and as float64 values [2][T][H][G][d] of the last layer."""
    n = c.d // c.gs * c.G if c.axis == 0 else c.d
    codes = torch.randint(0, 256, (c.layers, 2, c.T, c.heads, c.G, c.d * c.bits // 8), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.rand((c.layers, 2, c.T, c.heads, n), generator=g, device="cuda") * (0.3 if c.bits == 4 else 1.2) * c.spread
    m = (torch.rand(s.shape, generator=g, device="cuda") - 1.0) * 2.0 * c.spread
    meta = torch.stack([s, m], -1)
    if c.meta == "bf16":
        meta = meta.bfloat16()
    per = 8 // c.bits
    q = torch.stack([(codes[-1].long() >> (c.bits * i)) & (2 ** c.bits - 1) for i in range(per)], -1).reshape(2, c.T, c.heads, c.G, c.d).double()
    p = meta[-1].double()
    if c.axis == 0:
        p = p.reshape(2, c.T, c.heads, c.G, c.d // c.gs, 1, 2)
        x = (q.reshape(2, c.T, c.heads, c.G, c.d // c.gs, c.gs) * p[..., 0] + p[..., 1]).reshape(q.shape)
    else:
        p = p.reshape(2, c.T, c.heads, 1, c.d, 2)
        x = q * p[..., 0] + p[..., 1]
    return codes, meta, x


def expected(c, q, x, idx, rows, scale):
    """out, lse, and the bounds on both, in float64."""
    slots = [t for t in (idx.tolist() if idx is not None else range(c.k)) if 0 <= t < c.T]
    Hq = c.heads * c.repeat
    out = torch.zeros((Hq, c.t_q, c.d), dtype=torch.float64, device="cuda")
    tol, lse = out.clone(), torch.full((Hq, c.t_q), -math.inf, dtype=torch.float64, device="cuda")
    lse_tol = torch.zeros_like(lse)
    for i in range(Hq):
        h = i // c.repeat
        both = [torch.cat([rows["front"][kv][h].double(), x[kv][slots, h].reshape(-1, c.d), rows["recent"][kv][h].double()]) for kv in (0, 1)]
        dots = q[i].double() @ both[0].T * scale
        off = (q[i].double().abs() @ both[0].abs().T * abs(scale)).amax(-1, keepdim=True) * 2.0 ** -15 if both[0].shape[0] else torch.zeros((c.t_q, 1), device="cuda")
        if c.softcap:
            dots, off = c.softcap * torch.tanh(dots / c.softcap), off + c.softcap * 2.0 ** -20
        if c.causal:
            t, j = torch.arange(c.t_q, device="cuda")[:, None], torch.arange(c.recent, device="cuda")[None]
            dots[:, both[0].shape[0] - c.recent:].masked_fill_(j > t + c.recent - c.t_q, -math.inf)
        top = torch.logsumexp(dots, -1) if dots.shape[1] else torch.full((c.t_q,), -math.inf, device="cuda", dtype=torch.float64)
        p = torch.exp(dots - torch.where(top == -math.inf, 0.0, top)[:, None])
        out[i], lse[i] = p @ both[1], top
        tol[i] = (p @ both[1].abs()) * (2 * off + 2.0 ** -14)
        lse_tol[i] = off[:, 0] + 2.0 ** -20 * (1 + torch.where(top == -math.inf, 0.0, top).abs())
    return out, lse, tol, lse_tol


def check(oqm, c, stream=None, repeat=1):
    g = torch.Generator(device="cuda")
    g.manual_seed(c.seed)
    t = H.DT[c.dtype][1]
    codes, meta, x = stored(c, g)
    Hq = c.heads * c.repeat
    cfg = oqm.make_config(c.layers, c.heads, Hq, c.d, c.G, c.gs, c.T, qaxis=c.axis, bits=c.bits, in_dtype=H.DT[c.dtype][0],
                          out_dtype=H.DT[c.dtype][0], meta_dtype=H.DT[c.meta][0])
    h = oqm.tom_oqm_create(cfg)
    try:
        oqm.tom_oqm_bind(h, codes, meta, torch.empty(16, device="cuda"))
        oqm.tom_oqm_set_num_groups(h, c.T)
        # queries a token's heads beside each other, rows with room behind, outputs inside a larger buffer
        q = torch.randn((c.t_q, Hq, c.d), generator=g, device="cuda").to(t).transpose(0, 1)
        rows = {}
        for name, n in (("front", c.front), ("recent", c.recent)):
            rows[name] = [torch.randn((c.heads, n + 3, c.d), generator=g, device="cuda").to(t)[:, :n] for _ in range(2)]
        whole = torch.full((c.t_q, Hq + 1, c.d), 7.0, dtype=t, device="cuda")
        out = whole[:, :Hq].transpose(0, 1)
        lse = torch.full((Hq, c.t_q), 7.0, device="cuda")
        idx = None
        if not c.every:
            idx = torch.randint(0, c.T, (c.k,), generator=g, device="cuda").to(torch.int32)
            for i in range(c.holes):
                idx[(3 * i) % c.k] = (-1, c.T, 2 ** 31 - 1, -2 ** 31)[i % 4]
        scale = c.d ** -0.5
        n = c.front + c.k * c.G + c.recent
        ws = torch.empty(oqm.tom_oqm_attend_workspace_bytes(h, c.t_q, n), dtype=torch.uint8, device="cuda")
        ws.random_(0, 255)
        torch.cuda.synchronize()
        for _ in range(repeat):
            oqm.tom_oqm_attend(h, c.layers - 1, q, out, idx, c.k, rows["front"][0] if c.front else None, rows["front"][1] if c.front else None,
                               rows["recent"][0], rows["recent"][1], c.causal, None, c.softcap, lse, ws, stream)
        torch.cuda.synchronize()
    finally:
        oqm.tom_oqm_destroy(h)
    want, want_lse, tol, lse_tol = expected(c, q, x, idx, rows, scale)
    tol = tol + torch.finfo(t).eps / 2 * want.abs() + 1e-30
    off = (out.double() - want).abs()
    assert bool((off <= tol).all()), f"out is off by up to {float((off / tol).max())} times its bound"
    assert torch.equal(lse == -math.inf, want_lse == -math.inf)
    seen = want_lse != -math.inf
    assert bool((out[~seen] == 0).all())
    off = (lse.double() - want_lse).abs()[seen]
    assert bool((off <= lse_tol[seen]).all()), f"lse is off by up to {float((off / lse_tol[seen]).max())} times its bound"
    assert bool((whole[:, Hq] == 7.0).all()), "rows beside the output were written"


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d,gs", [(64, 32), (128, 64), (128, 8), (256, 128), (256, 32), (80, 16), (8, 8), (136, 8)])
def test_types_and_channels(oqm, dtype, d, gs):
    check(oqm, Case(dtype=dtype, d=d, gs=gs))


@pytest.mark.parametrize("axis,bits,meta,gs", [(a, b, m, gs) for a in (0, 1) for b in (4, 2) for m in ("f32", "bf16") for gs in ((16, 32, 128) if a == 0 else (64,))])
@pytest.mark.parametrize("t_q", [1, 40])
def test_storage_forms(oqm, axis, bits, meta, gs, t_q):
    check(oqm, Case(axis=axis, bits=bits, meta=meta, gs=gs, t_q=t_q, recent=50, seed=2))


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("G", [1, 2, 3, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 196])
def test_groups_that_end_inside_a_tile(oqm, G, axis):
    check(oqm, Case(G=G, axis=axis, T=11, k=7, holes=2, seed=G))


@pytest.mark.parametrize("t_q,repeat,heads", [(1, 1, 1), (1, 16, 1), (1, 17, 2), (2, 7, 4), (3, 5, 1), (5, 8, 2), (16, 1, 3), (17, 4, 1), (64, 7, 1), (130, 2, 2), (257, 1, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_queries(oqm, t_q, repeat, heads, dtype):
    check(oqm, Case(t_q=t_q, repeat=repeat, heads=heads, recent=t_q + 5, dtype=dtype, seed=t_q))


@pytest.mark.parametrize("front,k,recent,t_q", [
    (0, 0, 0, 1), (0, 0, 1, 1), (1, 0, 0, 1), (0, 1, 0, 1), (0, 0, 0, 5), (31, 0, 32, 3), (32, 2, 33, 2), (500, 0, 0, 2), (0, 0, 700, 60),
    (0, 0, 3, 8), (0, 0, 1, 20), (0, 4, 9, 20), (300, 3, 0, 4)])
@pytest.mark.parametrize("causal", [True, False])
def test_segments_and_rows_that_see_nothing(oqm, front, k, recent, t_q, causal):
    """With fewer recent rows than tokens, the first tokens of a causal call see none of them."""
    check(oqm, Case(front=front, k=k, recent=recent, t_q=t_q, causal=causal, seed=front + recent))


def test_holes_alone(oqm):
    for t_q in (1, 30):
        check(oqm, Case(k=4, holes=4, front=0, recent=0, t_q=t_q))
        check(oqm, Case(k=6, holes=4, front=0, recent=t_q, t_q=t_q))


@pytest.mark.parametrize("dtype,softcap", [("bf16", 30.0), ("bf16", 1.0), ("f16", 50.0), ("f32", 20.0), ("f32", 0.5)])
@pytest.mark.parametrize("t_q", [1, 33])
def test_capped_scores(oqm, dtype, softcap, t_q):
    check(oqm, Case(dtype=dtype, softcap=softcap, t_q=t_q, recent=40, seed=5))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("spread", [1e-3, 12.0])
def test_small_and_large_values(oqm, dtype, axis, spread):
    """A softmax that hardly tells rows apart, and one that a few rows make up."""
    check(oqm, Case(dtype=dtype, axis=axis, spread=spread, G=77, T=40, k=35))
    check(oqm, Case(dtype=dtype, axis=axis, spread=spread, G=77, T=40, k=9, t_q=20, recent=20))


@pytest.mark.parametrize("every,t_q,bits,axis", [(True, 1, 4, 0), (False, 1, 4, 0), (True, 1, 2, 0), (True, 1, 4, 1), (True, 9, 4, 0), (False, 70, 4, 0), (False, 70, 4, 1)])
def test_long_memories(oqm, every, t_q, bits, axis):
    check(oqm, Case(every=every, t_q=t_q, bits=bits, axis=axis, T=300, k=300, G=196, heads=1, recent=t_q + 3, layers=1, gs=64))


def test_stream_of_its_own_and_repeated_calls(oqm):
    check(oqm, Case(t_q=2), stream=torch.cuda.Stream(), repeat=3)


def test_graph_replays(oqm):
    """Captured, with new queries copied in and eager work between the replays; every replay equals the eager call."""
    c = Case(G=196, T=60, k=40, front=14, recent=20)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    codes, meta, _ = stored(c, g)
    Hq = c.heads * c.repeat
    cfg = oqm.make_config(c.layers, c.heads, Hq, c.d, c.G, c.gs, c.T)
    h = oqm.tom_oqm_create(cfg)
    oqm.tom_oqm_bind(h, codes, meta, torch.empty(16, device="cuda"))
    oqm.tom_oqm_set_num_groups(h, c.T)
    kv = [torch.randn((c.heads, 20, c.d), generator=g, device="cuda").bfloat16() for _ in range(4)]
    q, out, eager = (torch.empty((Hq, 1, c.d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    idx = torch.arange(0, 40, device="cuda", dtype=torch.int32)
    lse, eager_lse = (torch.empty((Hq, 1), device="cuda") for _ in range(2))
    ws, ws2 = (torch.empty(oqm.tom_oqm_attend_workspace_bytes(h, 1, 14 + 40 * 196 + 20), dtype=torch.uint8, device="cuda") for _ in range(2))

    def call(out, lse, ws):
        oqm.tom_oqm_attend(h, 1, q, out, idx, 40, kv[0][:, :14], kv[1][:, :14], kv[2], kv[3], lse=lse, workspace=ws)
    q.normal_(generator=g)
    call(out, lse, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, lse, ws)
    for _ in range(4):
        q.normal_(generator=g)
        call(eager, eager_lse, ws2)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(lse, eager_lse)
    oqm.tom_oqm_destroy(h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t_q", [1, 20])
def test_what_nobody_sees_may_be_anything(oqm, dtype, t_q):
    """NaN behind the last row of every view, in the pairs of groups that are not listed, in slots that holes would name, in
    keys behind a token's own; outputs stay finite and as they were."""
    t, H_k, R, d, G, T = H.DT[dtype][1], 2, 4, 128, 40, 6
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    cfg = oqm.make_config(1, H_k, H_k * R, d, G, 64, T + 2, in_dtype=H.DT[dtype][0], out_dtype=H.DT[dtype][0])
    h = oqm.tom_oqm_create(cfg)
    codes = torch.randint(0, 256, (1, 2, T + 2, H_k, G, d // 2), generator=g, device="cuda", dtype=torch.uint8)
    meta = torch.rand((1, 2, T + 2, H_k, G * 2, 2), generator=g, device="cuda")
    oqm.tom_oqm_bind(h, codes, meta, torch.empty(16, device="cuda"))
    oqm.tom_oqm_set_num_groups(h, T)
    rows = [torch.randn((H_k, 64, d), generator=g, device="cuda").to(t) for _ in range(4)]
    q = torch.randn((H_k * R, t_q, d), generator=g, device="cuda").to(t)
    idx = torch.tensor([4, -1, 1, T, 5], dtype=torch.int32, device="cuda")
    ws = torch.empty(oqm.tom_oqm_attend_workspace_bytes(h, t_q, 17 + 5 * G + 30), dtype=torch.uint8, device="cuda")
    got = []
    for spoil in (False, True):
        if spoil:
            for x in rows[:2]:
                x[:, 17:] = math.nan
            for x in rows[2:]:
                x[:, 30:] = math.nan
            for slot in (0, 2, 3, T, T + 1):
                meta[:, :, slot] = math.nan
            if t_q > 1:
                rows[2][:, 29] = math.nan        # the last token's own key: the others do not see it
        out = torch.zeros((H_k * R, t_q, d), dtype=t, device="cuda")
        lse = torch.zeros((H_k * R, t_q), device="cuda")
        oqm.tom_oqm_attend(h, 0, q, out, idx, 5, rows[0][:, :17], rows[1][:, :17], rows[2][:, :30], rows[3][:, :30], lse=lse, workspace=ws)
        torch.cuda.synchronize()
        got.append((out, lse))
    seen = slice(None) if t_q == 1 else slice(0, t_q - 1)
    assert bool(got[0][0].isfinite().all()) and bool(got[0][1].isfinite().all())
    assert torch.equal(got[0][0][:, seen], got[1][0][:, seen]) and torch.equal(got[0][1][:, seen], got[1][1][:, seen])
    oqm.tom_oqm_destroy(h)


@pytest.mark.parametrize("d,gs,bits,meta,G,dtype", [
    (128, 16, 4, "f32", 50, "bf16"), (128, 8, 2, "bf16", 33, "bf16"), (64, 16, 2, "f32", 7, "f16"), (256, 16, 4, "bf16", 40, "bf16"), (80, 8, 4, "f32", 31, "bf16"),
    (136, 8, 2, "f32", 64, "f16"), (8, 8, 2, "f32", 3, "bf16"), (96, 32, 4, "f32", 1, "bf16"), (128, 8, 4, "f32", 196, "f16")])
@pytest.mark.parametrize("t_q,causal", [(97, True), (300, False)])
def test_many_tokens_on_narrow_quant_groups(oqm, d, gs, bits, meta, G, dtype, t_q, causal):
    """More query rows than the reconstruction of a tile is shared by: 3 * t_q, over holes, a ragged front and recent rows."""
    check(oqm, Case(d=d, gs=gs, bits=bits, meta=meta, G=G, dtype=dtype, t_q=t_q, repeat=3, T=30, k=21, holes=3, front=45, recent=t_q + 17 if causal else 70,
                    causal=causal, softcap=25.0 if G == 50 else 0.0, seed=t_q + d))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bits", [4, 2])
@pytest.mark.parametrize("d,gs,axis", [(64, 32, 0), (64, 64, 0), (128, 32, 0), (128, 128, 0), (256, 32, 0), (256, 64, 0), (256, 128, 0), (64, 64, 1), (128, 64, 1), (256, 64, 1)])
def test_blocks_of_query_rows(oqm, d, gs, axis, bits, dtype):
    """More than 16 query rows: every compiled form, the last block ragged."""
    check(oqm, Case(d=d, gs=gs, axis=axis, bits=bits, dtype=dtype, t_q=31, recent=40, T=20, k=17, holes=2, seed=d + gs))


@pytest.mark.parametrize("axis", [0, 1])
@pytest.mark.parametrize("G", [1, 5, 31, 63, 64, 65, 130])
def test_groups_that_end_inside_a_shared_tile(oqm, G, axis):
    check(oqm, Case(G=G, axis=axis, T=11, k=9, holes=2, t_q=12, recent=12, seed=G))


def test_offsets_beyond_32_bits(oqm):
    """Slots more than 4 GiB into the storage, and rows half a GiB apart."""
    H_k, R, d, G, T = 4, 7, 128, 196, 90000
    g = torch.Generator(device="cuda")
    g.manual_seed(12)
    cfg = oqm.make_config(1, H_k, H_k * R, d, G, 64, T)
    codes = torch.empty((2, T, H_k, G, d // 2), dtype=torch.uint8, device="cuda")
    meta = torch.empty((2, T, H_k, G * 2, 2), device="cuda")
    slots = [3, T // 2, T - 1]
    for t in slots:
        codes[:, t] = torch.randint(0, 256, codes[:, t].shape, generator=g, device="cuda", dtype=torch.uint8)
        meta[:, t, ..., 0] = torch.rand((2, H_k, G * 2), generator=g, device="cuda") * 0.3
        meta[:, t, ..., 1] = torch.rand((2, H_k, G * 2), generator=g, device="cuda") * 2 - 2
    far = torch.empty((2, 9 << 28), dtype=torch.bfloat16, device="cuda")
    front = [x.as_strided((H_k, 9, d), (d, 1 << 28, 1)) for x in far]
    for x in front:
        x.normal_(generator=g)
    small = torch.stack([codes[:, t] for t in slots], 1), torch.stack([meta[:, t] for t in slots], 1)
    for t_q in (1, 9):
        q = torch.randn((H_k * R, t_q, d), generator=g, device="cuda").bfloat16()
        got = []
        for arrays, idx, rows, n in (((codes, meta), slots, front, T), (small, [0, 1, 2], [x.contiguous() for x in front], 3)):
            h = oqm.tom_oqm_create(oqm.make_config(1, H_k, H_k * R, d, G, 64, n))
            oqm.tom_oqm_bind(h, *arrays, torch.empty(16, device="cuda"))
            oqm.tom_oqm_set_num_groups(h, n)
            out, lse = torch.empty_like(q), torch.empty((H_k * R, t_q), device="cuda")
            ws = torch.empty(oqm.tom_oqm_attend_workspace_bytes(h, t_q, 9 + 3 * G), dtype=torch.uint8, device="cuda")
            oqm.tom_oqm_attend(h, 0, q, out, torch.tensor(idx, dtype=torch.int32, device="cuda"), 3, rows[0], rows[1], lse=lse, workspace=ws)
            torch.cuda.synchronize()
            oqm.tom_oqm_destroy(h)
            got.append((out, lse))
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1]) and bool(got[0][0].isfinite().all())
    # and moved: kept at the front, copied to the end of another
    h = oqm.tom_oqm_create(cfg)
    keys = torch.zeros((T, H_k, d), device="cuda")
    oqm.tom_oqm_bind(h, codes, meta, keys)
    oqm.tom_oqm_set_num_groups(h, T)
    oqm.tom_oqm_keep_groups(h, torch.tensor(slots, dtype=torch.int32, device="cuda"), 3)
    torch.cuda.synchronize()
    assert torch.equal(codes[:, :3], small[0]) and torch.equal(meta[:, :3], small[1])
    oqm.tom_oqm_set_num_groups(h, T - 3)
    oqm.tom_oqm_copy_groups(h, h, torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda"), 3)
    torch.cuda.synchronize()
    assert torch.equal(codes[:, T - 3:], small[0][:, [2, 0, 1]]) and torch.equal(meta[:, T - 3:], small[1][:, [2, 0, 1]])
    oqm.tom_oqm_destroy(h)


def test_negative_zero_and_other_scales(oqm):
    """scale below zero, zero, and as given; float32 and 16 bits."""
    for dtype in ("f32", "bf16"):
        for scale in (-0.07, 0.0, 0.25):
            t, H_k, R, d, G, T = H.DT[dtype][1], 1, 3, 64, 20, 4
            g = torch.Generator(device="cuda")
            g.manual_seed(5)
            c = Case(dtype=dtype, d=d, heads=H_k, repeat=R, G=G, gs=32, T=T, k=T, every=True, t_q=6, front=0, recent=9, layers=1)
            codes, meta, x = stored(c, g)
            h = oqm.tom_oqm_create(oqm.make_config(1, H_k, H_k * R, d, G, 32, T, in_dtype=H.DT[dtype][0], out_dtype=H.DT[dtype][0]))
            oqm.tom_oqm_bind(h, codes, meta, torch.empty(16, device="cuda"))
            oqm.tom_oqm_set_num_groups(h, T)
            q = torch.randn((H_k * R, 6, d), generator=g, device="cuda").to(t)
            recent = [torch.randn((H_k, 9, d), generator=g, device="cuda").to(t) for _ in range(2)]
            out, lse = torch.empty_like(q), torch.empty((H_k * R, 6), device="cuda")
            ws = torch.empty(oqm.tom_oqm_attend_workspace_bytes(h, 6, T * G + 9), dtype=torch.uint8, device="cuda")
            oqm.tom_oqm_attend(h, 0, q, out, None, T, recent_k=recent[0], recent_v=recent[1], scale=scale, lse=lse, workspace=ws)
            torch.cuda.synchronize()
            oqm.tom_oqm_destroy(h)
            none = torch.zeros((H_k, 0, d), device="cuda")
            want, want_lse, tol, lse_tol = expected(c, q, x, None, {"front": [none, none], "recent": recent}, scale)
            assert bool(((out.double() - want).abs() <= tol + want.abs() * torch.finfo(t).eps / 2).all())
            assert bool(((lse.double() - want_lse).abs() <= lse_tol).all())
