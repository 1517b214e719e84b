"""`Rotary` as a Python object: copies, pickles and changed configurations are what a call goes by (no GPU is touched: every call is
refused on the host, or has nothing to do)."""
import copy
import gc
import pickle

import pytest


@pytest.fixture()
def oqm():
    from paper_2510_18269_amd import oqm as m
    return m


def rotary(oqm):
    return oqm.Rotary(oqm.tom_oqm_rotary_t(64, 0, 0, 4096, 1e4, 1.0), 0x10000, 1.0)


def refused(oqm, rot, match):
    with pytest.raises(oqm.TomError, match=match):
        oqm.tom_oqm_rotate(rot, None)


@pytest.mark.parametrize("again", [copy.copy, copy.deepcopy, lambda r: pickle.loads(pickle.dumps(r))])
def test_copies_stand_alone(oqm, again):
    first = rotary(oqm)
    second = again(first)
    second.config = oqm.tom_oqm_rotary_t(64, 7, 0, 4096, 1e4, 1.0)
    refused(oqm, second, "layout")
    oqm.tom_oqm_rotate(first, None)                 # nothing to do: its own configuration is a good one
    third = again(first)
    del first, second
    gc.collect()
    oqm.tom_oqm_rotate(third, None)
    third.config.rotary_dim = 7
    refused(oqm, third, "rotary_dim 7")


def test_a_deep_copy_has_a_configuration_of_its_own(oqm):
    first = rotary(oqm)
    second = copy.deepcopy(first)
    second.config.rotary_dim = 9
    refused(oqm, second, "rotary_dim 9")
    oqm.tom_oqm_rotate(first, None)


def test_a_new_configuration_counts(oqm):
    rot = rotary(oqm)
    before = rot.config                             # alive, so that its place is not taken by the next one
    rot.config = oqm.tom_oqm_rotary_t(5, 0, 0, 4096, 1e4, 1.0)
    refused(oqm, rot, "rotary_dim 5")
    assert before.rotary_dim == 64
