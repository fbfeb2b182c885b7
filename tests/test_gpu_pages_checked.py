"""The paged cache's kernels under the checked build."""
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def fk():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


def test_small_cases_under_the_checked_build(fk):
    from paper_2507_20030_b200 import build
    env = dict(os.environ, FAEDKV_LIBRARY=build.build(debug=True))
    r = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "debug_build_pages_cases.py")], env=env, capture_output=True, text=True,
                       timeout=900)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "paged cases ok" in r.stdout
    assert fk.load().faedkv_debug_build() == 1 or fk.Pages(1, 1, 16, 1, 1, 1).debug_word() == 0


def test_the_word_of_no_handle(fk):
    assert fk.load().faedkv_pages_debug_word(None, None) == -1
