"""Attention where few rows carry the weight and the values lie in the others: every 32nd row is a sink, whose score stands `above` over
all else and whose value is zero, so that the outputs are the far tail of the softmax.

Tolerance: that of tests/test_gpu_attend.py, and half the last place that binary16 has for small numbers (2^-25): the outputs go down to
the smallest normal ones."""
import pytest
import torch

from tests import harness as H
from tests.test_gpu_attend import Case, expected
from tests.test_gpu_attend_large_scores import ROWS, call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def oqm():
    from paper_2510_18269_amd import oqm as m      # raises if the library is not built
    assert torch.cuda.is_available()
    return m


LEVELS = [("f16", 12.0), ("f16", 17.5), ("f16", 20.0), ("bf16", 20.0), ("f32", 20.0)]


def compare(c, got, q, x, rows):
    want, want_lse, tol, lse_tol = expected(c, q, x, None, rows, c.d ** -0.5)
    t = H.DT[c.dtype][1]
    tol = tol + torch.finfo(t).eps / 2 * want.abs() + 2.0 ** -25
    off = (got[0].double() - want).abs()
    assert bool((off <= tol).all()), f"out is off by up to {float((off / tol).max())} times its bound"
    off = (got[1].double() - want_lse).abs()
    assert bool((off <= lse_tol).all()), f"lse is off by up to {float((off / lse_tol).max())} times its bound"


def queries(c, g, t):
    """The first quant-group's channels are 2 in every query, the others small: what the sinks and the others differ by."""
    q = torch.randn((c.heads * c.repeat, c.t_q, c.d), generator=g, device="cuda") * 0.05
    q[..., :c.gs] = 2.0
    return q.to(t)


def sinks(c, above):
    return above / (2.0 * c.gs * c.d ** -0.5)   # of a sink's key in those channels


@pytest.mark.parametrize("shape", ROWS)
@pytest.mark.parametrize("dtype,above", LEVELS)
def test_rows_below_sinks(oqm, dtype, above, shape):
    n = 2048
    c = Case(dtype=dtype, heads=2, G=50, T=1, k=0, every=True, front=n, recent=0, causal=False, layers=1, **shape)
    t = H.DT[dtype][1]
    g = torch.Generator(device="cuda")
    g.manual_seed(c.d + c.t_q)
    q = queries(c, g, t)
    k = torch.randn((c.heads, n, c.d), generator=g, device="cuda") * 0.05
    v = 1000.0 * (1.0 + 0.3 * torch.randn((c.heads, n, c.d), generator=g, device="cuda"))
    k[..., :c.gs] = 0.0
    k[:, ::32, :c.gs] = sinks(c, above)
    v[:, ::32] = 0.0
    none = torch.zeros((c.heads, 0, c.d), dtype=t, device="cuda")
    rows = {"front": [k.to(t), v.to(t)], "recent": [none, none]}
    codes = torch.zeros(2 * c.heads * c.G * c.d // 2, dtype=torch.uint8, device="cuda")
    got = call(oqm, c, q, codes, torch.zeros(2 * c.heads * c.G * c.d * 2, device="cuda"), rows)
    compare(c, got, q, torch.zeros((2, 1, c.heads, c.G, c.d), dtype=torch.float64, device="cuda"), rows)


STORED = [dict(d=128, gs=64, t_q=1, repeat=7), dict(d=128, gs=32, t_q=60, repeat=7), dict(d=128, gs=128, t_q=1, repeat=7, axis=1), dict(d=64, gs=64, t_q=60, repeat=7, axis=1),
          dict(d=80, gs=16, t_q=5, repeat=4), dict(d=96, gs=32, t_q=5, repeat=4, axis=1), dict(d=128, gs=16, t_q=100, repeat=7), dict(d=256, gs=8, t_q=150, repeat=2)]


@pytest.mark.parametrize("shape", STORED)
@pytest.mark.parametrize("dtype,above", LEVELS)
def test_groups_below_sinks(oqm, dtype, above, shape):
    """A sink's key has the codes 15 in the first quant-group's channels, where all others have 0, and its value the codes 0."""
    G, T = 64, 16
    c = Case(dtype=dtype, heads=2, G=G, T=T, k=T, every=True, front=0, recent=0, causal=False, layers=1, **shape)
    t = H.DT[dtype][1]
    g = torch.Generator(device="cuda")
    g.manual_seed(c.d + c.t_q)
    q = queries(c, g, t)
    code = torch.randint(0, 16, (2, T, c.heads, G, c.d), generator=g, device="cuda")
    code[0, ..., :c.gs] = 0
    code[0, :, :, ::32, :c.gs] = 15
    code[1] = code[1].clamp(min=1)
    code[1, :, :, ::32] = 0
    n = c.d // c.gs * G if c.axis == 0 else c.d
    s = torch.full((2, T, c.heads, n), 0.003, device="cuda")
    s = s * (1.0 + torch.rand(s.shape, generator=g, device="cuda"))
    if c.axis == 0:
        s[0].view(T, c.heads, G, c.d // c.gs)[..., 0] = sinks(c, above) / 15.0
    else:
        s[0][..., :c.gs] = sinks(c, above) / 15.0
    s[1] *= 15000.0
    meta = torch.stack([s, torch.zeros_like(s)], -1)
    x = code.double().view(2, T, c.heads, G, c.d)
    p = s.double()
    x = x * (p.view(2, T, c.heads, G, c.d // c.gs, 1).expand(-1, -1, -1, -1, -1, c.gs).reshape(x.shape) if c.axis == 0 else p.view(2, T, c.heads, 1, c.d))
    codes = (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8)
    none = torch.zeros((c.heads, 0, c.d), dtype=t, device="cuda")
    rows = {"front": [none, none], "recent": [none, none]}
    got = call(oqm, c, q, codes, meta, rows)
    compare(c, got, q, x, rows)
