"""The binding reads tensors as the PyTorch it was built against lays them out, and refuses to be loaded beside another."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LOAD = "import torch.version\nimport sys\nif len(sys.argv) > 1: torch.version.__version__ = sys.argv[1]\nimport paper_2510_18269_amd.oqm\nprint('loaded')"


def load(*version):
    return subprocess.run([sys.executable, "-c", LOAD, *version], cwd=ROOT, capture_output=True, text=True, timeout=120)


def test_the_pytorch_it_was_built_against():
    import torch
    assert load().stdout.strip() == "loaded" and load(torch.__version__).stdout.strip() == "loaded"


def test_another_pytorch():
    for other in ("2.10.0", "2.9.1+rocm7.0", ""):
        r = load(other)
        assert r.returncode != 0 and "ImportError" in r.stderr and f"cannot be used with {other}" in r.stderr and "build" in r.stderr
