"""What the training calls ask of their caller in memory (CPU)."""
import ctypes

import pytest

from paper_2507_02006_amd import _binding as B_


@pytest.mark.parametrize("dtype,size", [(B_.DTYPE_F32, 4), (B_.DTYPE_BF16, 2), (B_.DTYPE_F16, 2)])
@pytest.mark.parametrize("t", [1, 100, 4096])
def test_cross_entropy_workspace_does_not_grow_with_the_table(t, dtype, size):
    """Some GB for a table of 100 GB: what is kept of each row and tile of the
    table, a piece of packed rows and one of dz."""
    need, d, v = ctypes.c_int64(), 512, (100 << 30) // (512 * size)
    for grads in (0, 1):
        assert B_.load().aires_linear_xent_workspace(t, d, v, dtype, grads, ctypes.byref(need)) == B_.OK
        assert need.value < (3 << 30) + 8 * t * (v // 256 + 1), need.value
