"""Calls beyond what a launch or an index holds are refused on the host as UNSUPPORTED, before anything is queued (no GPU is touched)."""
import pytest
import torch

from tests.test_operator_refusals import Fake


@pytest.fixture()
def oqm():
    from paper_2510_18269_amd import oqm as m
    return m


def unsupported(oqm, match, call):
    with pytest.raises(oqm.TomError, match=match) as e:
        call()
    assert e.value.status == oqm.TOM_ERR_UNSUPPORTED


# 2^30 query rows are 2^32 lanes where a wave takes 16 of them, and where a workgroup of 256 lanes takes 64; 2^31 rows are where one of
# 512 takes 256
@pytest.mark.parametrize("dtype,kv_heads,q_heads,t_q,d,gs", [
    (torch.float32, 1024, 1024, 2 ** 20, 8, 8), (torch.float32, 1, 2047, 2 ** 20, 8, 8), (torch.bfloat16, 1, 1024, 2 ** 20, 64, 32),
    (torch.bfloat16, 1, 2047, 2 ** 20, 256, 16), (torch.float16, 4, 1024, 2 ** 20, 128, 128)])
def test_attend_of_more_lanes_than_a_grid(oqm, dtype, kv_heads, q_heads, t_q, d, gs):
    code = {torch.float32: oqm.TOM_F32, torch.bfloat16: oqm.TOM_BF16, torch.float16: oqm.TOM_F16}[dtype]
    h = oqm.tom_oqm_create(oqm.make_config(1, kv_heads, q_heads, d, 16, gs, 8, in_dtype=code, out_dtype=code))
    try:
        q, rows = Fake((q_heads, t_q, d), dtype), Fake((kv_heads, 64, d), dtype)
        unsupported(oqm, "lanes", lambda: oqm.tom_oqm_attend(h, 0, q, q, recent_k=rows, recent_v=rows, causal=False))
    finally:
        oqm.tom_oqm_destroy(h)


# a lane takes two elements at odd addresses, 16 bytes and up to four heads elsewhere; a head of 2 channels has one lane
@pytest.mark.parametrize("rows,heads,d,n,address", [(2 ** 20, 256, 128, 128, 0x10002), (2 ** 20, 512, 128, 128, 0x10002), (2 ** 27, 1, 2048, 2048, 0x10002),
                                                    (2 ** 23, 128, 256, 256, 0x10000), (2 ** 20, 2047, 64, 64, 0x10004)])
def test_rotate_of_more_lanes_than_a_grid(oqm, rows, heads, d, n, address):
    rot = oqm.Rotary(oqm.tom_oqm_rotary_t(n, 0, 0, 4096, 1e4, 1.0), 0x10000, 1.0)
    x = Fake((rows, heads, d), address=address)
    unsupported(oqm, "lanes", lambda: oqm.tom_oqm_rotate(rot, 0x10000, q=x, q_out=x))


def test_attend_of_more_rows_than_an_index(oqm):
    """2^31 - 4097 rows of keys: the limit that the header gives, one more is refused."""
    most = 2 ** 31 - 4097
    h = oqm.tom_oqm_create(oqm.make_config(1, 1, 1, 64, 1, 32, 8))
    oqm.tom_oqm_bind(h, 0x100000, 0x200000, 0x300000)
    try:
        q = Fake((1, 1, 64))
        for front, recent, k in ((most + 1, 0, 0), (most - 4, 3, 2), (5, most - 4, 0), (0, 0, most + 1)):
            f, r = Fake((1, front, 64)), Fake((1, recent, 64))
            unsupported(oqm, f"{most + 1} rows: at most {most}", lambda: oqm.tom_oqm_attend(h, 0, q, q, 0x10000, k, f, f, r, r))
        need = oqm.tom_oqm_attend_workspace_bytes(h, 1, most)
        assert need > 0 and oqm.tom_oqm_attend_workspace_bytes(h, 1, most + 1) == 0
        f = Fake((1, most, 64))
        with pytest.raises(oqm.TomError, match=f"workspace of {need} bytes needed"):     # as many are taken
            oqm.tom_oqm_attend(h, 0, q, q, front_k=f, front_v=f)
    finally:
        oqm.tom_oqm_destroy(h)
