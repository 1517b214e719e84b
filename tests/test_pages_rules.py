"""The rules of the attention over pages that go by numbers alone, built for the host under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU is used)."""
import os

from tests.test_sanitizers import SAN, _host_build


def test_rules_at_the_ends_of_their_ranges(tmp_path):
    assert "pages rules driver: clean" in _host_build(str(tmp_path / "pages_rules_driver"), os.path.join(SAN, "pages_rules_driver.cpp"))
