"""Every form of the 8-bit linear layer captured by its first call in a fresh process (tests/int8_first_capture_child.py)."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_first_calls_in_a_fresh_process_are_captured():
    r = subprocess.run([sys.executable, "-u", os.path.join(ROOT, "tests", "int8_first_capture_child.py")], capture_output=True, text=True,
                       timeout=300, cwd=ROOT)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert r.stdout.strip().endswith("ok")
