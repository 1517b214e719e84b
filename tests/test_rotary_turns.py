"""The angles that a `Rotary` holds are read as rotary_dim / 2 float64 numbers: a tensor that is something else is refused (no GPU is
touched)."""
import pytest
import torch

from tests.test_operator_refusals import Fake


@pytest.fixture()
def oqm():
    from paper_2510_18269_amd import oqm as m
    return m


def rotary(oqm, turns, rotary_dim=64):
    return oqm.Rotary(oqm.tom_oqm_rotary_t(rotary_dim, 0, 0, 4096, 1e4, 1.0), turns, 1.0)


@pytest.mark.parametrize("turns", [
    Fake((31,), torch.float64), Fake((0,), torch.float64), Fake((32,), torch.float32), Fake((64,), torch.float32), Fake((32,), torch.int64),
    Fake((32,), torch.bfloat16), Fake((32,), torch.float64, (2,)), Fake((32,), torch.float64, is_cuda=False), torch.zeros(32, dtype=torch.float64)])
def test_turns_that_are_not_the_angles(oqm, turns):
    t = Fake((3, 2, 64))
    with pytest.raises(AssertionError):
        oqm.tom_oqm_rotate(rotary(oqm, turns), Fake((3,), torch.int64), q=t, q_out=t)


def test_turns_that_are(oqm):
    """These reach the library, which finds nothing to do, or a stride that it refuses."""
    far = Fake((3, 2, 64), strides=(2 ** 41, 64, 1))
    for turns in (Fake((32,), torch.float64), Fake((40,), torch.float64), 0x10000):
        oqm.tom_oqm_rotate(rotary(oqm, turns), None)
        with pytest.raises(oqm.TomError, match="strides"):
            oqm.tom_oqm_rotate(rotary(oqm, turns), Fake((3,), torch.int64), q=far, q_out=far)
    with pytest.raises(oqm.TomError, match="rotary_dim"):
        oqm.tom_oqm_rotate(rotary(oqm, Fake((32,), torch.float64), -6), None)


def test_a_rotary_that_is_refused_takes_no_memory(oqm):
    import tracemalloc
    for n in (2 ** 24, 2050, -2 ** 24):
        tracemalloc.start()
        with pytest.raises(oqm.TomError, match="rotary_dim"):
            oqm.tom_oqm_rotary_turns(oqm.tom_oqm_rotary_t(n, 0, 0, 4096, 1e4, 1.0))
        assert tracemalloc.get_traced_memory()[1] < 2 ** 20
        tracemalloc.stop()
    assert len(oqm.tom_oqm_rotary_turns(oqm.tom_oqm_rotary_t(2048, 0, 0, 4096, 1e4, 1.0))[0]) == 1024
