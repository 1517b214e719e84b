"""AddressSanitizer + UndefinedBehaviorSanitizer pass over the host side of the calls on pages, and the rules that cut the attention over them against the
counts that its workgroups work out (no GPU is used)."""
import os

from tests.test_sanitizers import ROOT, SAN, _host_build


def test_host_side_and_cuts_are_clean(tmp_path):
    csrc = os.path.join(ROOT, "paper_2510_18269_amd", "csrc")
    out = _host_build(str(tmp_path / "pages_driver"), *(os.path.join(csrc, f) for f in ("oqm_api.hip", "oqm_attend_pages_api.hip", "oqm_draft.hip")),
                      os.path.join(SAN, "pages_driver.cpp"))
    assert "pages driver: clean" in out
