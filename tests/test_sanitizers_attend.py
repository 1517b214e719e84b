"""AddressSanitizer + UndefinedBehaviorSanitizer pass over the attention's rules at the ends of their ranges (no GPU is used)."""
import os

from tests.test_sanitizers import SAN, _host_build


def test_rules_at_the_ends_of_their_ranges(tmp_path):
    assert "attend driver: clean" in _host_build(str(tmp_path / "attend_driver"), os.path.join(SAN, "attend_driver.cpp"))
