"""Rotary positions, head norms and the copy of values (`tom_oqm_rotate`) against their formulas in float64.

Tolerance of a turned channel: the cosine and sine carry 2^-22, the products and their sum 2^-23, a norm 2^-21 of the value,
together under 2^-20 of |a| + |b|, and half a step of the output's type."""
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


def turned(x, w, positions, radians, amplitude, layout, n, eps):
    """float64 [T][heads][d] and the sum |a| + |b| of every channel's pair."""
    x = x.double()
    if w is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w.double()
    half = torch.arange(n // 2, device="cuda")
    one, two = (half, half + n // 2) if layout == 0 else (2 * half, 2 * half + 1)
    angle = positions.double()[:, None] * radians[None]
    c, s = amplitude * torch.cos(angle)[:, None], amplitude * torch.sin(angle)[:, None]
    y, size = x.clone(), x.abs()
    a, b = x[..., one], x[..., two]
    y[..., one], y[..., two] = a * c - b * s, b * c + a * s
    size[..., one] = size[..., two] = amplitude * (a.abs() + b.abs())
    return y, size


def check(oqm, dtype, d, n, layout, T, Hq, Hk, norm, values, first=0, scaling=0, factor=1.0, shift=0, by_heads=False, in_place=False):
    g = torch.Generator(device="cuda")
    g.manual_seed(T * 7 + d + n)
    t = H.DT[dtype][1]
    rot = oqm.Rotary.create(n, layout, 10000.0, scaling, factor, 4096)
    sizes = (Hq, Hk, Hk)
    # `shift` elements in front of every row: other alignments of the vectors
    whole = torch.randn((T, sum(sizes), d + shift), generator=g, device="cuda").to(t)[..., shift:]
    if by_heads:
        whole = whole.transpose(0, 1).contiguous().transpose(0, 1)
    x = list(whole.split(sizes, 1))
    ref = [v.clone() for v in x]
    room = [torch.full((T + 2, heads, d + shift), 5.0, dtype=t, device="cuda") for heads in sizes]
    out = x if in_place else [r[1:-1, :, shift:] for r in room]
    w = [(1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(t) for _ in range(2)] if norm else [None, None]
    positions = first + torch.randint(0, 3 * T + 1, (T,), generator=g, device="cuda")
    kw = dict(q=x[0], q_out=out[0]) if Hq else {}
    if values:
        kw.update(v=x[2], v_out=out[2])
    oqm.tom_oqm_rotate(rot, positions, k=x[1], k_out=out[1], q_norm=w[0] if Hq else None, k_norm=w[1], norm_eps=1e-5, **kw)
    torch.cuda.synchronize()
    radians = torch.tensor(oqm.tom_oqm_rotary_turns(rot.config)[0], dtype=torch.float64, device="cuda") * 2 * math.pi
    # the angle itself is a float64 product: 2^-51 of it
    slack = 2.0 ** -20 + float(positions.abs().max() if T else 0) * 2.0 ** -51
    for i in ((0, 1) if Hq else (1,)):
        want, size = turned(ref[i], w[i], positions, radians, rot.amplitude, layout, n, 1e-5)
        off = (out[i].double() - want).abs()
        tol = size * slack + torch.finfo(t).eps / 2 * want.abs() + torch.finfo(t).smallest_normal
        assert bool((off <= tol).all()), f"side {i}: off by up to {float((off / tol).max())} times the bound"
    if values:
        assert torch.equal(out[2], ref[2])
    if not in_place:
        for i in range(3):
            r = room[i]
            assert bool((r[0] == 5).all()) and bool((r[-1] == 5).all()) and bool((r[..., :shift] == 5).all())
            if (i == 0 and not Hq) or (i == 2 and not values):
                assert bool((r == 5).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("d,n", [(128, 128), (64, 64), (80, 80), (96, 48), (256, 256), (128, 64), (128, 6), (128, 2), (256, 130), (2, 2), (66, 64), (128, 126), (512, 512), (2048, 2048), (2046, 1026)])
@pytest.mark.parametrize("norm", [False, True])
def test_shapes_of_a_head(oqm, dtype, layout, d, n, norm):
    check(oqm, dtype, d, n, layout, 5, 4, 2, norm, True)


@pytest.mark.parametrize("T,Hq,Hk,by_heads", [(1, 28, 4, False), (1, 1, 1, False), (2, 0, 3, True), (333, 28, 4, False), (700, 0, 56, True), (1000, 16, 8, False), (3000, 8, 8, True)])
@pytest.mark.parametrize("norm", [False, True])
def test_sizes(oqm, T, Hq, Hk, by_heads, norm):
    check(oqm, "bf16", 128, 128, 0, T, Hq, Hk, norm, Hq > 0, by_heads=by_heads, first=12000)


@pytest.mark.parametrize("shift", [1, 2, 4, 6])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [0, 1])
def test_alignments(oqm, shift, dtype, layout):
    check(oqm, dtype, 64, 64, layout, 9, 4, 2, True, True, shift=shift)


@pytest.mark.parametrize("first", [0, 10 ** 6, 2 ** 31 + 5, 10 ** 12, -77])
@pytest.mark.parametrize("layout", [0, 1])
def test_far_and_negative_positions(oqm, first, layout):
    check(oqm, "f32", 64, 64, layout, 40, 2, 1, False, True, first=first)


@pytest.mark.parametrize("scaling", [0, 1, 2, 3, 4])
def test_scalings(oqm, scaling):
    check(oqm, "f32", 128, 96, 0, 30, 3, 1, True, True, first=70000, scaling=scaling, factor=8.0)


@pytest.mark.parametrize("layout", [0, 1])
def test_in_place(oqm, layout):
    check(oqm, "bf16", 128, 64, layout, 50, 6, 2, True, True, in_place=True)


def test_no_rows_and_no_sides(oqm):
    check(oqm, "bf16", 64, 64, 0, 0, 2, 1, False, True)
    rot = oqm.Rotary.create(64)
    oqm.tom_oqm_rotate(rot, None)
    v, out = torch.randn(3, 2, 64, device="cuda"), torch.zeros(3, 2, 64, device="cuda")
    oqm.tom_oqm_rotate(rot, None, v=v, v_out=out)       # values alone need no positions
    torch.cuda.synchronize()
    assert torch.equal(v, out)
