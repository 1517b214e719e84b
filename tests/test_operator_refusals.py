"""What the rotary, the attention over stored groups and the moves of groups refuse on the host, before anything is
launched, and what they take without work (no GPU is touched)."""
import ctypes as C
import math

import pytest
import torch

from tests.test_binding import FakeTensor


class Fake(FakeTensor):
    """A device tensor by its shape: contiguous unless strides are given."""
    def __init__(self, shape, dtype=torch.bfloat16, strides=None, address=0x10000, is_cuda=True):
        n, out = 1, []
        for s in reversed(shape):
            out.insert(0, n)
            n *= s
        super().__init__(tuple(strides or out), is_cuda, n)
        self.shape, self.dtype, self.address, self.flat = tuple(shape), dtype, address, strides is None
    def data_ptr(self): return self.address
    def element_size(self): return self.dtype.itemsize
    def is_contiguous(self): return self.flat


@pytest.fixture()
def oqm():
    from paper_2510_18269_amd import oqm as m
    return m


@pytest.fixture()
def store(oqm):
    h = oqm.tom_oqm_create(oqm.make_config(2, 2, 6, 64, 16, 32, 8))
    oqm.tom_oqm_bind(h, 0x100000, 0x200000, 0x300000)
    oqm.tom_oqm_set_num_groups(h, 5)
    yield h
    oqm.tom_oqm_destroy(h)


def refuses(oqm, match, call, status=None):
    with pytest.raises(oqm.TomError, match=match) as e:
        call()
    assert e.value.status == (oqm.TOM_ERR_INVALID_ARG if status is None else status)


# ---- rotary ----------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("field,value", [
    ("rotary_dim", 0), ("rotary_dim", 7), ("rotary_dim", 2050), ("rotary_dim", -2), ("layout", 2), ("layout", -1), ("scaling", 5), ("scaling", -1),
    ("original_length", 0), ("base", 1.0), ("base", math.nan), ("base", math.inf), ("base", -5.0), ("factor", 0.5), ("factor", math.nan), ("factor", math.inf)])
def test_bad_rotaries(oqm, field, value):
    kw = dict(rotary_dim=64, layout=0, scaling=0, original_length=4096, base=10000.0, factor=1.0)
    kw[field] = value
    refuses(oqm, field, lambda: oqm.tom_oqm_rotary_turns(oqm.tom_oqm_rotary_t(**kw)))


def test_base_scaling_needs_two_pairs(oqm):
    refuses(oqm, "TOM_ROTARY_BASE", lambda: oqm.Rotary.create(2, scaling=oqm.TOM_ROTARY_BASE, device="cpu"))


@pytest.mark.parametrize("n", [2, 4, 64, 96, 128])
@pytest.mark.parametrize("factor,original", [(1.0, 4096), (8.0, 4096), (32.0, 8192), (2.5, 1)])
def test_turns_follow_their_formulas(oqm, n, factor, original):
    """In decimals of 50 digits, from the definitions: float64 rounds a handful of times (16 half steps are allowed)."""
    from decimal import Decimal, getcontext
    getcontext().prec = 50
    base, fac = Decimal(500000), Decimal(factor)
    pi = Decimal("3.14159265358979323846264338327950288419716939937510")
    for scaling in range(5):
        if scaling == oqm.TOM_ROTARY_BASE and n < 4:
            continue
        turns, amplitude = oqm.tom_oqm_rotary_turns(oqm.tom_oqm_rotary_t(n, 0, scaling, original, 500000.0, factor))
        assert len(turns) == n // 2
        b = base * (fac.ln() * n / (n - 2)).exp() if scaling == oqm.TOM_ROTARY_BASE else base
        place = lambda r: n * (Decimal(original) / (r * 2 * pi)).ln() / (2 * b.ln())  # noqa: E731
        lo, hi = max(math.floor(place(32)), 0), min(math.ceil(place(1)), n - 1)
        for i in range(n // 2):
            f = (b.ln() * (Decimal(-2 * i) / n)).exp()
            kept = Decimal(1)
            if scaling == oqm.TOM_ROTARY_LINEAR:
                kept = Decimal(0)
            elif scaling == oqm.TOM_ROTARY_BY_PARTS:
                kept = 1 - min(max(Decimal(i - lo) / max(Decimal(hi - lo), Decimal("0.001")), Decimal(0)), Decimal(1))
            elif scaling == oqm.TOM_ROTARY_BY_WAVELENGTH:
                kept = min(max((original * f / (2 * pi) - 1) / 3, Decimal(0)), Decimal(1))
            want = (f * kept + f / fac * (1 - kept)) / (2 * pi)
            # `kept` is a difference: its error counts against the plain frequency
            assert abs(turns[i] - float(want)) <= 16 * 2.0 ** -53 * (float(want) + float(f) / 6.28 * (0 if kept in (0, 1) else 8))
        want = 0.1 * math.log(factor) + 1 if scaling == oqm.TOM_ROTARY_BY_PARTS else 1.0
        assert abs(amplitude - want) <= 2.0 ** -23


def test_rotate_refuses(oqm):
    rot = oqm.Rotary(oqm.tom_oqm_rotary_t(64, 0, 0, 4096, 1e4, 1.0), 0x10000, 1.0)
    pos = Fake((3,), torch.int64)
    t = lambda *shape, **kw: Fake(shape or (3, 2, 64), **kw)  # noqa: E731
    refuses(oqm, "both", lambda: oqm.tom_oqm_rotate(rot, pos, q=t()))
    refuses(oqm, "both", lambda: oqm.tom_oqm_rotate(rot, pos, v_out=t()))
    refuses(oqm, "agree", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(), q_out=t(3, 3, 64)))
    refuses(oqm, "agree", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(), q_out=t(), k=t(2, 2, 64), k_out=t(2, 2, 64)))
    refuses(oqm, "agree", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(), q_out=t(dtype=torch.float16)))
    refuses(oqm, "channels", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(3, 2, 62), q_out=t(3, 2, 62)))
    refuses(oqm, "channels", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(3, 2, 2050), q_out=t(3, 2, 2050)))
    refuses(oqm, "aligned", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(address=0x10001), q_out=t()))
    refuses(oqm, "strides", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(strides=(2 ** 41, 64, 1)), q_out=t()))
    refuses(oqm, "overlap", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(), q_out=t(strides=(0, 64, 1))))
    refuses(oqm, "overlap", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(), q_out=t(strides=(128, 32, 1))))
    refuses(oqm, "norm weights", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(), q_out=t(), k_norm=0x10000))
    refuses(oqm, "norm_eps", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(), q_out=t(), norm_eps=math.nan))
    refuses(oqm, "norm_eps", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(), q_out=t(), norm_eps=-1.0))
    refuses(oqm, "positions", lambda: oqm.tom_oqm_rotate(rot, None, q=t(), q_out=t()))
    refuses(oqm, "data", lambda: oqm.tom_oqm_rotate(rot, pos, q=t(address=0), q_out=t()))
    huge = Fake((2 ** 27, 16, 64))
    refuses(oqm, "2\\^31", lambda: oqm.tom_oqm_rotate(rot, 0x10000, q=huge, q_out=huge), oqm.TOM_ERR_UNSUPPORTED)
    for call in (lambda: oqm.tom_oqm_rotate(rot, Fake((2,), torch.int64), q=t(), q_out=t()),        # too few positions
                 lambda: oqm.tom_oqm_rotate(rot, Fake((3,), torch.int32), q=t(), q_out=t()),
                 lambda: oqm.tom_oqm_rotate(rot, Fake((3,), torch.int64, (2,)), q=t(), q_out=t()),
                 lambda: oqm.tom_oqm_rotate(rot, pos, q=t(is_cuda=False), q_out=t()),
                 lambda: oqm.tom_oqm_rotate(rot, pos, q=0x10000, q_out=t()),
                 lambda: oqm.tom_oqm_rotate(rot, pos, q=t(2, 64), q_out=t()),
                 lambda: oqm.tom_oqm_rotate(rot, pos, q=t(strides=(128, 1, 2)), q_out=t()),
                 lambda: oqm.tom_oqm_rotate(rot, pos, q=t(dtype=torch.int32), q_out=t()),
                 lambda: oqm.tom_oqm_rotate(rot, pos, q=t(dtype=torch.float64), q_out=t()),
                 lambda: oqm.tom_oqm_rotate(rot, pos, q=t(), q_out=t(), q_norm=Fake((63,))),
                 lambda: oqm.tom_oqm_rotate(rot, pos, q=t(), q_out=t(), q_norm=Fake((64,), torch.float32))):
        with pytest.raises(AssertionError):
            call()
    # nothing to do
    oqm.tom_oqm_rotate(rot, None)
    oqm.tom_oqm_rotate(rot, None, q=t(0, 2, 64), q_out=t(0, 2, 64))
    oqm.tom_oqm_rotate(rot, None, q=t(3, 0, 64), q_out=t(3, 0, 64))


# ---- attention -------------------------------------------------------------------------------------------------------


def test_attend_refuses(oqm, store):
    def call(**kw):
        a = dict(h=store, layer=0, q=Fake((6, 3, 64)), out=Fake((6, 3, 64)), idx=Fake((4,), torch.int32), k_eff=4, recent_k=Fake((2, 3, 64)),
                 recent_v=Fake((2, 3, 64)), workspace=Fake((1 << 20,), torch.uint8))
        a.update(kw)
        oqm.tom_oqm_attend(**a)
    refuses(oqm, "handle is NULL", lambda: call(h=None))
    refuses(oqm, "layer", lambda: call(layer=2))
    refuses(oqm, "layer", lambda: call(layer=-1))
    refuses(oqm, "q and out", lambda: call(out=None))
    refuses(oqm, "q and out", lambda: call(q=None))
    refuses(oqm, "k_eff", lambda: call(idx=None, k_eff=6))
    refuses(oqm, "k_eff", lambda: call(k_eff=-1))
    refuses(oqm, "out_dtype", lambda: call(q=Fake((6, 3, 64), torch.float16)))
    refuses(oqm, "out_dtype", lambda: call(front_k=Fake((2, 3, 64), torch.float32), front_v=Fake((2, 3, 64), torch.float32)))
    refuses(oqm, "out is", lambda: call(out=Fake((6, 4, 64))))
    refuses(oqm, "q is", lambda: call(q=Fake((4, 3, 64))))
    refuses(oqm, "recent_k is", lambda: call(recent_k=Fake((3, 3, 64))))
    refuses(oqm, "same rows", lambda: call(recent_v=Fake((2, 4, 64))))
    refuses(oqm, "same rows", lambda: call(front_k=Fake((2, 4, 64))))
    refuses(oqm, "16 bytes", lambda: call(q=Fake((6, 3, 64), address=0x10008)))
    refuses(oqm, "16 bytes", lambda: call(recent_v=Fake((2, 3, 64), strides=(204, 68, 1))))
    refuses(oqm, "overlap", lambda: call(out=Fake((6, 3, 64), strides=(0, 64, 1))))
    refuses(oqm, "overlap", lambda: call(out=Fake((6, 3, 64), strides=(192, 32, 1))))
    refuses(oqm, "scale", lambda: call(scale=math.nan))
    refuses(oqm, "softcap", lambda: call(softcap=-1.0))
    refuses(oqm, "softcap", lambda: call(softcap=math.inf))
    need = oqm.tom_oqm_attend_workspace_bytes(store, 3, 4000 * 16 + 3)
    assert need > 0
    many = dict(k_eff=4000, idx=0x10000)
    refuses(oqm, f"{need} bytes needed, {need - 1} given", lambda: call(**many, workspace=Fake((need - 1,), torch.uint8)))
    refuses(oqm, "0 given", lambda: call(**many, workspace=None))
    refuses(oqm, "aligned", lambda: call(**many, workspace=Fake((need,), torch.uint8, address=0x10008)))
    refuses(oqm, "rows", lambda: call(k_eff=2 ** 27, idx=0x10000), oqm.TOM_ERR_UNSUPPORTED)
    refuses(oqm, "new tokens", lambda: call(q=Fake((6, 2 ** 20 + 1, 64)), out=Fake((6, 2 ** 20 + 1, 64))), oqm.TOM_ERR_UNSUPPORTED)
    for kw in (dict(idx=Fake((3,), torch.int32)), dict(idx=Fake((4,), torch.int64)), dict(lse=Fake((17,), torch.float32)),
               dict(lse=Fake((6, 3), torch.bfloat16)), dict(q=Fake((6, 3, 64), is_cuda=False)), dict(q=Fake((6, 64)))):
        with pytest.raises(AssertionError):
            call(**kw)
    call(q=Fake((6, 0, 64)), out=Fake((6, 0, 64)))      # no tokens: nothing launched
    other = oqm.tom_oqm_create(oqm.make_config(2, 2, 6, 64, 16, 32, 8))
    refuses(oqm, "bind", lambda: call(h=other), oqm.TOM_ERR_NOT_BOUND)
    oqm.tom_oqm_destroy(other)
    wide = oqm.tom_oqm_create(oqm.make_config(1, 1, 1, 264, 4, 8, 8))
    refuses(oqm, "256", lambda: call(h=wide, k_eff=0), oqm.TOM_ERR_UNSUPPORTED)
    oqm.tom_oqm_destroy(wide)


def test_attend_workspace_grows_with_the_rows(oqm, store):
    for t_q in (1, 2, 7, 64, 1000):
        sizes = [oqm.tom_oqm_attend_workspace_bytes(store, t_q, n) for n in (0, 1, 31, 64, 65, 200, 5000, 10 ** 5, 10 ** 6, 2 ** 31 - 5000)]
        assert sizes == sorted(sizes)
    for bad in ((0, 10), (-1, 10), (2 ** 20 + 1, 10), (1, -1), (1, 2 ** 40)):
        assert oqm.tom_oqm_attend_workspace_bytes(store, *bad) == 0
    assert oqm.tom_oqm_attend_workspace_bytes(None, 1, 10) == 0


# ---- groups ----------------------------------------------------------------------------------------------------------


def test_keep_refuses(oqm, store):
    idx = Fake((5,), torch.int32)
    refuses(oqm, "handle is NULL", lambda: oqm.tom_oqm_keep_groups(None, idx, 1))
    refuses(oqm, "outside", lambda: oqm.tom_oqm_keep_groups(store, 0x10000, 6))
    refuses(oqm, "outside", lambda: oqm.tom_oqm_keep_groups(store, idx, -1))
    refuses(oqm, "idx", lambda: oqm.tom_oqm_keep_groups(store, None, 2))
    refuses(oqm, "aligned", lambda: oqm.tom_oqm_keep_groups(store, 0x10002, 2))
    with pytest.raises(AssertionError):
        oqm.tom_oqm_keep_groups(store, Fake((5,), torch.int64), 2)
    with pytest.raises(AssertionError):
        oqm.tom_oqm_keep_groups(store, Fake((1,), torch.int32), 2)
    with pytest.raises(C.ArgumentError):
        oqm.tom_oqm_keep_groups(store, idx, 1.5)
    assert oqm.tom_oqm_num_groups(store) == 5           # a refused call has changed nothing
    oqm.tom_oqm_keep_groups(store, None, 0)
    assert oqm.tom_oqm_num_groups(store) == 0
    bare = oqm.tom_oqm_create(oqm.make_config(2, 2, 6, 64, 16, 32, 8))
    refuses(oqm, "bind", lambda: oqm.tom_oqm_keep_groups(bare, None, 0), oqm.TOM_ERR_NOT_BOUND)
    oqm.tom_oqm_destroy(bare)


def test_copy_refuses(oqm, store):
    idx = Fake((9,), torch.int32)
    base = dict(n_layers=2, n_kv_heads=2, n_q_heads=6, head_dim=64, group_tokens=16, qgroup=32, capacity_groups=8)
    handles = []

    def other(at=0x1000000, **kw):
        h = oqm.tom_oqm_create(oqm.make_config(**{**base, **kw}))
        oqm.tom_oqm_bind(h, at, at + 0x100000, at + 0x200000)
        handles.append(h)
        return h
    try:
        for kw in (dict(n_layers=1), dict(n_kv_heads=1), dict(head_dim=128), dict(group_tokens=15), dict(qgroup=16), dict(bits=2),
                   dict(qaxis=oqm.TOM_QAXIS_TOKENS), dict(meta_dtype=oqm.TOM_BF16)):
            refuses(oqm, "different shapes", lambda: oqm.tom_oqm_copy_groups(other(**kw), store, idx, 1))
        good = other(n_q_heads=2, capacity_groups=4, in_dtype=oqm.TOM_F16)      # the queries' heads and dtypes do not matter
        refuses(oqm, "handle is NULL", lambda: oqm.tom_oqm_copy_groups(good, None, idx, 1))
        refuses(oqm, "n < 0", lambda: oqm.tom_oqm_copy_groups(good, store, idx, -1))
        refuses(oqm, "idx", lambda: oqm.tom_oqm_copy_groups(good, store, None, 1))
        refuses(oqm, "capacity", lambda: oqm.tom_oqm_copy_groups(good, store, idx, 5), oqm.TOM_ERR_CAPACITY)
        refuses(oqm, "capacity", lambda: oqm.tom_oqm_copy_groups(store, store, idx, 4), oqm.TOM_ERR_CAPACITY)
        refuses(oqm, "overlap", lambda: oqm.tom_oqm_copy_groups(other(at=0x100800), store, idx, 1))
        # a second handle of the same storage, behind which groups of the first would be written over
        same = oqm.tom_oqm_create(oqm.make_config(**base))
        handles.append(same)
        oqm.tom_oqm_bind(same, 0x100000, 0x200000, 0x300000)
        refuses(oqm, "overlap", lambda: oqm.tom_oqm_copy_groups(same, store, idx, 1))
        oqm.tom_oqm_copy_groups(good, store, None, 0)
        assert oqm.tom_oqm_num_groups(good) == 0 and oqm.tom_oqm_num_groups(store) == 5
        bare = oqm.tom_oqm_create(oqm.make_config(**base))
        handles.append(bare)
        refuses(oqm, "bind", lambda: oqm.tom_oqm_copy_groups(bare, store, idx, 1), oqm.TOM_ERR_NOT_BOUND)
    finally:
        for h in handles:
            oqm.tom_oqm_destroy(h)
