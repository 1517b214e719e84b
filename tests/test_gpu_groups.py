"""Groups kept and copied as they are stored (`tom_oqm_keep_groups`, `tom_oqm_copy_groups`): every byte of all three arrays."""
import pytest
import torch

from tests import harness as H

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def oqm():
    from paper_2510_18269_amd import oqm as m      # raises if the library is not built
    assert torch.cuda.is_available()
    return m


def memory(oqm, seed, T, capacity, L=2, heads=2, d=64, G=5, gs=16, bits=4, axis=0, meta="f32"):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    mem = oqm.Memory.allocate(oqm.make_config(L, heads, heads, d, G, gs, capacity, qaxis=axis, bits=bits, meta_dtype=H.DT[meta][0]))
    for x in (mem.codes, mem.meta, mem.keys):
        x.view(torch.uint8).random_(0, 255, generator=g)
    oqm.tom_oqm_set_num_groups(mem.handle, T)
    return mem


def planes(mem):
    """The three arrays as bytes [plane][slot][bytes of a slot]."""
    c = mem.cfg
    return [x.view(torch.uint8).reshape(c.n_layers * n, c.capacity_groups, -1) for x, n in ((mem.codes, 2), (mem.meta, 2), (mem.keys, 1))]


SHAPES = [dict(), dict(L=1, heads=1, d=8, G=1, gs=8, bits=2), dict(L=1, heads=1, d=8, G=1, gs=8), dict(L=3, heads=1, d=24, G=7, gs=8, bits=2, meta="bf16"),
          dict(heads=4, d=128, G=196, gs=64), dict(L=1, heads=3, d=72, G=11, axis=1, meta="bf16"), dict(L=1, heads=1, d=16, G=3, gs=8, bits=2),
          dict(L=2, heads=1, d=16, G=3, gs=16)]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("T,n", [(1, 1), (9, 0), (9, 9), (40, 1), (40, 39), (300, 150), (2500, 2000)])
def test_keep(oqm, shape, T, n):
    if T > 300 and shape.get("G", 5) > 11:
        T, n = 400, 333
    mem = memory(oqm, T + n, T, T + 3, **shape)
    try:
        before = [x.clone() for x in planes(mem)]
        g = torch.Generator().manual_seed(n)
        idx = torch.randperm(T, generator=g)[:n].sort().values.to(torch.int32).cuda()
        torch.cuda.synchronize()
        oqm.tom_oqm_keep_groups(mem.handle, idx, n)
        torch.cuda.synchronize()
        assert mem.n_groups == n
        for x, y in zip(planes(mem), before):
            assert torch.equal(x[:, :n], y[:, idx.long()])
            assert torch.equal(x[:, n:], y[:, n:])       # what is dropped, or was free, is not touched
    finally:
        mem.close()


def test_keep_leaves_slots_of_indices_outside(oqm):
    mem = memory(oqm, 3, 12, 16)
    try:
        before = [x.clone() for x in planes(mem)]
        idx = torch.tensor([-5, 2, 3, 12, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
        oqm.tom_oqm_keep_groups(mem.handle, idx, 5)
        torch.cuda.synchronize()
        for x, y in zip(planes(mem), before):
            assert torch.equal(x[:, 1], y[:, 2]) and torch.equal(x[:, 2], y[:, 3])
            assert torch.equal(x[:, 0], y[:, 0]) and torch.equal(x[:, 3:], y[:, 3:])
    finally:
        mem.close()


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("T,n,into", [(1, 1, 0), (9, 0, 4), (9, 20, 4), (300, 150, 31)])
def test_copy(oqm, shape, T, n, into):
    src, dst = memory(oqm, T, T, T + 2, **shape), memory(oqm, T + 1, into, into + n + 5, **shape)
    try:
        was, before = [x.clone() for x in planes(src)], [x.clone() for x in planes(dst)]
        g = torch.Generator().manual_seed(n)
        idx = torch.randint(0, T, (n,), generator=g).to(torch.int32)
        if n > 3:
            idx[1], idx[2] = -1, T
        dev = idx.cuda()
        torch.cuda.synchronize()
        oqm.tom_oqm_copy_groups(dst.handle, src.handle, dev, n)
        torch.cuda.synchronize()
        assert dst.n_groups == into + n and src.n_groups == T
        for s, x, y in zip(planes(src), planes(dst), before):
            want = y.clone()
            for i, t in enumerate(idx.tolist()):
                if 0 <= t < T:
                    want[:, into + i] = s[:, t]
            assert torch.equal(x, want)
        assert all(torch.equal(a, b) for a, b in zip(planes(src), was))
    finally:
        src.close()
        dst.close()


def test_copy_within_a_memory(oqm):
    mem = memory(oqm, 8, 10, 25, d=128, G=50, gs=64)
    try:
        before = [x.clone() for x in planes(mem)]
        idx = torch.tensor([9, 0, 0, 5], dtype=torch.int32, device="cuda")
        oqm.tom_oqm_copy_groups(mem.handle, mem.handle, idx, 4)
        torch.cuda.synchronize()
        assert mem.n_groups == 14
        for x, y in zip(planes(mem), before):
            assert torch.equal(x[:, :10], y[:, :10]) and torch.equal(x[:, 10:14], y[:, idx.long()]) and torch.equal(x[:, 14:], y[:, 14:])
    finally:
        mem.close()


def test_kept_and_copied_groups_are_retrieved_as_before(oqm):
    """What a fork or a shortened memory retrieves is what the original gives for the same groups."""
    mem, fork = memory(oqm, 5, 30, 40, d=64, G=16, gs=32), memory(oqm, 6, 0, 40, d=64, G=16, gs=32)
    try:
        mem.meta.copy_(torch.rand_like(mem.meta))
        keep = torch.tensor([0, 3, 4, 11, 29], dtype=torch.int32, device="cuda")
        rows = torch.arange(5, dtype=torch.int32, device="cuda")
        out = [torch.zeros((2, 2, 5 * 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(6)]
        oqm.tom_oqm_dequant_gather(mem.handle, 0, 2, keep.repeat(2, 1), 5, 5, out[0], out[1])
        oqm.tom_oqm_copy_groups(fork.handle, mem.handle, keep, 5)
        oqm.tom_oqm_keep_groups(mem.handle, keep, 5)
        oqm.tom_oqm_dequant_gather(mem.handle, 0, 2, rows.repeat(2, 1), 5, 5, out[2], out[3])
        oqm.tom_oqm_dequant_gather(fork.handle, 0, 2, rows.repeat(2, 1), 5, 5, out[4], out[5])
        torch.cuda.synchronize()
        for i in (2, 4):
            assert torch.equal(out[0], out[i]) and torch.equal(out[1], out[i + 1])
    finally:
        mem.close()
        fork.close()
