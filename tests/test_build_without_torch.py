"""The C ABI needs no torch: neither to be built nor to be loaded (no GPU)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("torch", ["None", "types.SimpleNamespace(version=types.SimpleNamespace(cuda=None))"])
def test_build_and_load(torch):
    """Without torch, and with one that has no CUDA: the library is built and loads, and the operators on
    torch tensors say what they miss."""
    code = (f"import sys, types; sys.modules['torch'] = {torch}\n"
            "from paper_1905_12948_gb300 import build, load\n"
            "from paper_1905_12948_gb300.build import _tokens_command, nvcc\n"
            "assert _tokens_command(nvcc(), 'x') is None\n"
            "assert build.build() == build.LIB\n"
            "assert load().gmc_strerror(1)\n")
    p = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert p.returncode == 0, p.stderr
