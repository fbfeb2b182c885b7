"""The kernels of shared pages and differential attention under the checked build."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_small_cases_under_the_checked_build():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2507_20030_b200 import build
    env = dict(os.environ, FAEDKV_LIBRARY=build.build(debug=True))
    r = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "debug_build_share_cases.py")], env=env, capture_output=True, text=True,
                       timeout=900)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "cases of shared pages ok" in r.stdout
