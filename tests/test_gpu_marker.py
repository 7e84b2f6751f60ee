"""Tests that need a GPU are skipped, not failed, where there is none, whether or not their file says so itself."""
import os
import subprocess
import sys

import pytest

from gpu_util import has_gpu

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(has_gpu(), reason="with a GPU they run")
def test_marked_tests_are_skipped_without_a_gpu():
    run = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", "test_gpu_second_derivatives.py"],
                         cwd=HERE, capture_output=True, text=True, timeout=110)
    assert run.returncode == 0 and "2 skipped" in run.stdout, run.stdout[-2000:]
