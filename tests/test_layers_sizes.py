"""Sizes at the ends of their ranges, in the calls that need no GPU (CPU)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

NO_ROWS = """
import ctypes
from paper_2507_02006_amd import _binding as B_
lib, need, v, top = B_.load(), ctypes.c_int64(-1), %d, %d
assert lib.aires_log_probs_workspace(0, v, top, ctypes.byref(need)) == B_.OK and need.value == 0
for Z in (B_.Dense(0, v, v, 0, 0, None), B_.Dense(0, v, v, 2, 0, 4096)):
    z = ctypes.byref(Z)
    assert lib.aires_log_probs(z, None, 0, top, None, None, None, None, None, None, 0, None) == B_.OK
    assert lib.aires_log_probs_backward(z, None, 0, None, None, None, None, z, None) == B_.OK
"""


@pytest.mark.parametrize("v", [1, 2048, 2049, 100000, 2 ** 30 - 1])
@pytest.mark.parametrize("top", [0, 1, 64])
def test_log_probs_of_no_rows(v, top):
    """No rows need no workspace and are no error, however many classes (a process of its
    own: one that divides by the number of rows ends)."""
    r = subprocess.run([sys.executable, "-c", NO_ROWS % (v, top)], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])
