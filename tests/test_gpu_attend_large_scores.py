"""Attention with scores so large that float32 rounds them: one row of keys stands far above the others, and its value comes out."""
import math

import pytest
import torch

from tests import harness as H
from tests.test_gpu_attend import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def oqm():
    from paper_2510_18269_amd import oqm as m      # raises if the library is not built
    assert torch.cuda.is_available()
    return m


def call(oqm, c, q, codes, meta, rows, scale=None):
    t = H.DT[c.dtype]
    h = oqm.tom_oqm_create(oqm.make_config(1, c.heads, c.heads * c.repeat, c.d, c.G, c.gs, max(1, c.T), qaxis=c.axis, in_dtype=t[0], out_dtype=t[0]))
    try:
        oqm.tom_oqm_bind(h, codes, meta, torch.empty(16, device="cuda"))
        oqm.tom_oqm_set_num_groups(h, c.T)
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        n = c.front + c.k * c.G + c.recent
        ws = torch.empty(oqm.tom_oqm_attend_workspace_bytes(h, c.t_q, n), dtype=torch.uint8, device="cuda")
        oqm.tom_oqm_attend(h, 0, q, out, None, c.k, *rows["front"], *rows["recent"], causal=c.causal, scale=scale, lse=lse, workspace=ws)
        torch.cuda.synchronize()
    finally:
        oqm.tom_oqm_destroy(h)
    return out, lse


# general, folded and shared forms, by head_dim, quant-group and rows
ROWS = [dict(d=128, gs=64, t_q=1, repeat=7), dict(d=64, gs=32, t_q=1, repeat=3), dict(d=128, gs=64, t_q=60, repeat=7), dict(d=256, gs=64, t_q=20, repeat=7),
        dict(d=80, gs=16, t_q=5, repeat=4), dict(d=192, gs=8, t_q=3, repeat=2), dict(d=128, gs=16, t_q=100, repeat=7), dict(d=256, gs=8, t_q=150, repeat=2)]


@pytest.mark.parametrize("shape", ROWS)
@pytest.mark.parametrize("dtype,size", [("f16", 1500.0), ("f16", 8000.0), ("f16", 16000.0), ("bf16", 16000.0), ("bf16", 3e5), ("bf16", 1e8), ("f32", 1e8)])
def test_scores_that_float32_rounds(oqm, dtype, size, shape):
    """Scores of 2^21 to 2^55.  The general, the folded and the shared form; 16 rows of queries and more."""
    n = 200
    c = Case(dtype=dtype, heads=2, G=50, T=1, k=0, every=True, front=n, recent=0, causal=False, layers=1, **shape)
    t = H.DT[dtype][1]
    g = torch.Generator(device="cuda")
    g.manual_seed(c.d + c.t_q + int(size))
    q = (torch.randn((c.heads * c.repeat, c.t_q, c.d), generator=g, device="cuda").clamp(-4, 4) * size).to(t)
    k, v = ((torch.randn((c.heads, n, c.d), generator=g, device="cuda").clamp(-4, 4) * by).to(t) for by in (size, 1.0))
    none = torch.zeros((c.heads, 0, c.d), dtype=t, device="cuda")
    rows = {"front": [k, v], "recent": [none, none]}
    codes = torch.zeros(2 * c.heads * c.G * c.d // 2, dtype=torch.uint8, device="cuda")
    out, lse = call(oqm, c, q, codes, torch.zeros(2 * c.heads * c.G * c.d * 2, device="cuda"), rows)
    assert bool(out.isfinite().all()) and bool(lse.isfinite().all())
    for i in range(c.heads * c.repeat):
        dots = q[i].double() @ k[i // c.repeat].double().T * c.d ** -0.5
        top = dots.topk(2, -1)
        # float32 sums of d products: 2^-24 * d of the largest sum of magnitudes, and the score itself rounded
        off = (q[i].double().abs() @ k[i // c.repeat].double().abs().T).amax(-1) * c.d ** -0.5 * (c.d + 8) * 2.0 ** -24
        clear = top.values[:, 0] - top.values[:, 1] > 2 * off + 20.0
        assert torch.equal(out[i][clear], v[i // c.repeat][top.indices[:, 0]][clear])
        assert bool(((lse[i].double() - top.values[:, 0]).abs() <= off + math.log(n) + 1.0).all())
