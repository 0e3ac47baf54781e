"""The library and torch share one HIP runtime, whichever is asked for first
(no GPU needed)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("first", ["import torch; lif.load()", "lif.load(); import torch", "lif.lif_version(); import torch"])
def test_one_hip_runtime(first):
    code = ("import paper_2603_13283_amd as lif; " + first +
            "; print(len({l.split()[-1] for l in open('/proc/self/maps') if 'libamdhip64' in l}))")
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr
    assert out.stdout.split()[-1] == "1"
