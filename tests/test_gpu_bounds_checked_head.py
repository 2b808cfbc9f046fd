"""The tests of the operators around the LM head once more against the bounds-checking build of the library (see
test_gpu_bounds_checked.py): they must pass as before, and the kernels must count no violation."""
import os
import subprocess
import sys

import pytest

from paper_2509_08721_b200 import build

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FILES = ["tests/test_gpu_preference.py", "tests/test_gpu_norm.py", "tests/test_gpu_preference_step.py", "tests/test_gpu_norm_long.py"]


def test_operators_pass_and_count_no_violation_in_the_checked_build(tmp_path):
    lib = build.build(checked=True)
    report = tmp_path / "violations.txt"
    env = dict(os.environ, SAPO_B200_LIB=lib, SAPO_BOUNDS_REPORT=str(report))
    res = subprocess.run([sys.executable, "-m", "pytest", *FILES, "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider"],
                         cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stdout[-3000:] + res.stderr[-2000:]
    assert report.read_text() == "0"
