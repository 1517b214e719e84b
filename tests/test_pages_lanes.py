"""The calls on pages run on the host, lane by lane, under AddressSanitizer: what numbers on the device that make no sense lead to (no GPU is used)."""
import os

from tests.test_sanitizers import ROOT, SAN, _run

CSRC = os.path.join(ROOT, "paper_2510_18269_amd", "csrc")


def clean(tmp_path, driver, *sources):
    # the compiler of the kernels, for the host alone: it has their vector types; the folder with the host's hip_runtime.h stands in front of the real one
    exe = str(tmp_path / driver)
    _run([os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++"), "-x", "c++", "-O2", "-g", "-std=c++17", "-fsanitize=address", "-w",
          "-I", os.path.join(SAN, "lanes"), "-I", CSRC, "-I", os.path.join(ROOT, "include"),
          os.path.join(SAN, driver + ".cpp"), *(os.path.join(CSRC, s) for s in sources), "-o", exe])
    assert "driver: clean" in _run([exe], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0:detect_stack_use_after_return=0"))


def test_numbers_are_never_trusted_with_an_address(tmp_path):
    clean(tmp_path, "pages_lanes_driver", "oqm_attend_pages_api.hip")


def test_trees_appended_and_kept_rows_stay_inside(tmp_path):
    clean(tmp_path, "rows_lanes_driver")
