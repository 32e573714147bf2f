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


def test_refusals_of_the_calls_with_a_rest():
    """As the calls without it (CPU: each fails before anything is launched)."""
    import ctypes

    from paper_2507_02006_amd import _binding as B_
    lib, fake = B_.load(), 4096
    Z, other = B_.Dense(3, 50, 50, 0, 0, fake), B_.Dense(3, 50, 50, 0, 0, 8192)

    def forward(Z=Z, lse=fake, rest=fake, top=0):
        return lib.aires_log_probs_rest(ctypes.byref(Z), None, 0, top, None, None, lse, rest, None, None, None, 0, None)

    def back(Z=Z, lse=fake, h=fake, dZ=other, labels=fake):
        return lib.aires_log_probs_backward_rest(ctypes.byref(Z), labels, 0, lse, fake, h, fake, fake, ctypes.byref(dZ), None)

    assert forward(lse=None) == forward(top=65) == forward(top=3) == forward(Z=B_.Dense(3, 50, 7, 0, 0, fake)) == B_.E_INVALID_ARG
    assert forward(Z=B_.Dense(3, 0, 0, 0, 0, fake)) == B_.E_DIM
    assert back(lse=None) == back(h=None) == back(labels=None) == back(dZ=B_.Dense(3, 50, 51, 0, 0, fake)) == B_.E_INVALID_ARG
    assert back(dZ=B_.Dense(3, 51, 51, 0, 0, 8192)) == B_.E_DIM
    none = B_.Dense(0, 50, 50, 0, 0, None)
    assert forward(Z=none) == back(Z=none, dZ=none) == B_.OK
