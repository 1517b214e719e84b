"""Attention along the tokens over values in which code * scale and zero nearly cancel: all codes are 15 and a zero -15 * scale * (1 + 2^-12 r).

The two meet in the same two parts of the probabilities, so that what the parts leave of them (2^-17) moves only the value that remains.
Tolerance: 2^-16 of the value; 2^-20 of its zero (products and sums in float32, a handful of roundings of 2^-24); 2^-18 of the scale for codes
in the upper half of a byte, 2^-14 in the lower half, where the matrix cores cut off places of sub-normal numbers; the scores' 2^-15 of
sum_c |q_c k_c| twice over the value; half a step of the output's type, no less than 2^-25 in binary16."""
import pytest
import torch

from tests import harness as H

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def oqm():
    from paper_2510_18269_amd import oqm as m      # raises if the library is not built
    assert torch.cuda.is_available()
    return m


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("t_q,G", [(1, 2), (1, 7), (60, 3), (60, 8)])
def test_values_that_cancel(oqm, dtype, d, t_q, G):
    heads, repeat = 4, 7
    t = H.DT[dtype]
    g = torch.Generator(device="cuda")
    g.manual_seed(d + t_q + G)
    s = torch.rand((2, 1, heads, d), generator=g, device="cuda") + 0.5
    m = -15.0 * s * (1 + 2.0 ** -12 * torch.randn(s.shape, generator=g, device="cuda"))
    code = torch.full((2, 1, heads, G, d), 15, device="cuda")
    s[0], m[0], code[0] = 0.02, -0.15, torch.randint(0, 16, code[0].shape, generator=g, device="cuda")      # keys: small and all different
    codes = (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8)
    pairs = torch.stack([s, m], -1)
    h = oqm.tom_oqm_create(oqm.make_config(1, heads, heads * repeat, d, G, 32, 1, qaxis=oqm.TOM_QAXIS_TOKENS, in_dtype=t[0], out_dtype=t[0]))
    try:
        oqm.tom_oqm_bind(h, codes, pairs, torch.empty(16, device="cuda"))
        oqm.tom_oqm_set_num_groups(h, 1)
        q = torch.randn((heads * repeat, t_q, d), generator=g, device="cuda").to(t[1])
        out = torch.empty_like(q)
        ws = torch.empty(oqm.tom_oqm_attend_workspace_bytes(h, t_q, G), dtype=torch.uint8, device="cuda")
        oqm.tom_oqm_attend(h, 0, q, out, None, 1, scale=1.0, workspace=ws)
        torch.cuda.synchronize()
    finally:
        oqm.tom_oqm_destroy(h)
    x = (code.double() * s.double()[..., None, :] + m.double()[..., None, :])[:, 0]      # [2][H][G][d]
    place = torch.where(torch.arange(d, device="cuda") % 2 == 0, 2.0 ** -14, 2.0 ** -18)
    for i in range(heads * repeat):
        n = i // repeat
        y = q[i].double()
        p = torch.softmax(y @ x[0, n].T, -1)
        off = (y.abs() @ x[0, n].abs().T).amax(-1, keepdim=True) * 2.0 ** -15
        want = p @ x[1, n]
        tol = (2.0 ** -16 + 2 * off) * (p @ x[1, n].abs()) + 2.0 ** -20 * m[1, 0, n].abs().double() + place * s[1, 0, n].double()
        tol = tol + (torch.finfo(t[1]).eps / 2 * want.abs()).clamp(min=2.0 ** -25 if dtype == "f16" else 0.0)
        apart = (out[i].double() - want).abs()
        assert bool((apart <= tol).all()), f"off by up to {float((apart / tol).max())} times its bound"
