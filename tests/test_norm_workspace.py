"""The workspace of the norm's backward pass has room in front of its sums for the 256 bytes that other calls keep in theirs (no GPU needed: the pointers are fake)."""
import ctypes as C

import pytest

from paper_2602_06183_b200 import binding, build


@pytest.mark.parametrize("T,D", [(1, 8), (5, 64), (148, 1408), (3000, 4096), (1 << 28, 32768)])
def test_head_is_left(T, D):
    build.build()
    need = binding.sf_rmsnorm_bwd_workspace_size(T, D)
    assert need == 256 + 4 * min(T, 148) * D
    at = [C.c_void_p((i + 1) << 46) for i in range(8)]        # far from one another
    assert binding.lib().sf_rmsnorm_bwd(at[0], at[1], at[2], at[3], None, T, D, at[4], at[5], at[6], need - 256, None) == binding.SF_ERR_WORKSPACE
