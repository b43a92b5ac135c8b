"""The library and the native product calls are built where torch is not installed, as a caller with raw addresses wants them; the module on torch tensors is left out."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SCRIPT = """
import sys
sys.modules["torch"] = None  # an import of it fails
from paper_1805_10692_amd import build
calls = []
build.subprocess.check_call = lambda cmd: calls.append(cmd)
build.os.replace = lambda a, b: calls.append(b)
build.build_library(verbose=False)
print(sum(c == build.LIB for c in calls), sum(c == build.NATIVE_BINDING for c in calls), sum(c == build.NATIVE_OPERATORS for c in calls))
"""


def test_build_without_torch():
    out = subprocess.run([sys.executable, "-c", SCRIPT], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert out.returncode == 0, out.stderr[-500:]
    assert "torch is not installed" in out.stdout
    assert out.stdout.splitlines()[-1] == "1 1 0"
