"""The example that runs the operators together on what the tier moves, as a user would run it."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_hybrid_decode_example():
    r = subprocess.run([sys.executable, os.path.join(ROOT, "examples", "hybrid_decode.py")], cwd=ROOT,
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr
    print("\n" + r.stdout.strip())
    assert "decode bit-exact" in r.stdout
