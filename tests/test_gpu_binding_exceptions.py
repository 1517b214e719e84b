"""Tensors that have no storage, sizes or strides raise in every call that reads them, and leave the process alive."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def oqm():
    from paper_2510_18269_amd import oqm as m      # raises if the library is not built
    assert torch.cuda.is_available()
    return m


@pytest.fixture(scope="module")
def odd():
    """Two nested tensors of three dimensions (the second of whole numbers), and a sparse one."""
    nested = torch.nested.nested_tensor([torch.zeros(2, 64, device="cuda"), torch.zeros(3, 64, device="cuda")])
    whole = torch.nested.nested_tensor([torch.zeros(2, 4, dtype=torch.int32, device="cuda"), torch.zeros(3, 4, dtype=torch.int32, device="cuda")])
    return [nested, whole, torch.zeros((4, 2, 64), device="cuda").to_sparse()]


def raises(call):
    with pytest.raises((RuntimeError, AssertionError)):
        call()


def test_odd_tensors(oqm, odd):
    rot = oqm.Rotary.create(64)
    t = torch.zeros((2, 2, 64), device="cuda")
    at = torch.zeros(2, dtype=torch.int64, device="cuda")
    mem = oqm.Memory.allocate(oqm.make_config(1, 2, 2, 64, 4, 32, 8, in_dtype=oqm.TOM_F32, out_dtype=oqm.TOM_F32))
    idx = torch.zeros(4, dtype=torch.int32, device="cuda")
    h = mem.handle
    oqm.tom_oqm_set_num_groups(h, 4)
    try:
        for x in odd:
            raises(lambda: oqm.tom_oqm_rotate(rot, at, q=x, q_out=t))
            raises(lambda: oqm.tom_oqm_rotate(rot, at, k=t, k_out=x))
            raises(lambda: oqm.tom_oqm_rotate(rot, x, q=t, q_out=t))
            raises(lambda: oqm.tom_oqm_rotate(rot, at, q=t, q_out=t, q_norm=x))
            raises(lambda: oqm.tom_oqm_rotate(oqm.Rotary(rot.config, x, 1.0), at, q=t, q_out=t))
            raises(lambda: oqm.tom_oqm_attend(h, 0, x, t, recent_k=t, recent_v=t))
            raises(lambda: oqm.tom_oqm_attend(h, 0, t, x, recent_k=t, recent_v=t))
            raises(lambda: oqm.tom_oqm_attend(h, 0, t, t, recent_k=x, recent_v=t))
            raises(lambda: oqm.tom_oqm_attend(h, 0, t, t, idx=x, k_eff=100, recent_k=t, recent_v=t))
            raises(lambda: oqm.tom_oqm_attend(h, 0, t, t, recent_k=t, recent_v=t, lse=x))
            raises(lambda: oqm.tom_oqm_keep_groups(h, x, 100))
            raises(lambda: oqm.tom_oqm_copy_groups(h, h, x, 100))
        raises(lambda: oqm.tom_oqm_attend(h, 0, t, t, idx=idx, k_eff=4, recent_k=t, recent_v=t, workspace=odd[2]))
        assert mem.n_groups == 4
        torch.cuda.synchronize()
    finally:
        mem.close()
