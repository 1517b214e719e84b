"""The attention over pages run on the host, lane by lane, under AddressSanitizer: what numbers on the device that make no sense lead to (no GPU is used)."""
import os

from tests.test_sanitizers import ROOT, SAN, _run


def test_numbers_are_never_trusted_with_an_address(tmp_path):
    exe, csrc = str(tmp_path / "pages_lanes_driver"), os.path.join(ROOT, "paper_2510_18269_amd", "csrc")
    # the compiler of the kernels, for the host alone: it has their vector types; the folder with the host's hip_runtime.h stands in front of the real one
    _run([os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++"), "-x", "c++", "-O2", "-g", "-std=c++17", "-fsanitize=address", "-w",
          "-I", os.path.join(SAN, "lanes"), "-I", csrc, "-I", os.path.join(ROOT, "include"),
          os.path.join(SAN, "pages_lanes_driver.cpp"), os.path.join(csrc, "oqm_attend_pages_api.hip"), "-o", exe])
    out = _run([exe], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0:detect_stack_use_after_return=0"))
    assert "pages lanes driver: clean" in out
