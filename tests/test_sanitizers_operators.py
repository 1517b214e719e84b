"""AddressSanitizer + UndefinedBehaviorSanitizer pass over the host side of the rotary, the attention over stored groups and the
moves of groups (no GPU is used)."""
import os

from tests.test_sanitizers import ROOT, SAN, _host_build


def test_host_validation_is_clean_under_asan_and_ubsan(tmp_path):
    csrc = os.path.join(ROOT, "paper_2510_18269_amd", "csrc")
    out = _host_build(str(tmp_path / "operators_driver"), *(os.path.join(csrc, f) for f in ("oqm_api.hip", "oqm_attend_api.hip", "oqm_rotate.hip", "oqm_groups.hip")),
                      os.path.join(SAN, "operators_driver.cpp"))
    assert "operators sanitizer driver: clean" in out
