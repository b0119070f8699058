"""The package before torch: one HIP runtime in the process, whichever a program imports first."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("order", ["paper_2409_12517_amd, torch", "torch, paper_2409_12517_amd"])
def test_one_runtime(order):
    code = f"import {order}\nprint(*sorted({{l.split()[-1] for l in open('/proc/self/maps') if 'libamdhip64' in l}}))"
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    assert len(out.stdout.split()) == 1, out.stdout
