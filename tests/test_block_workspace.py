"""The joins' workspace has a bound whatever the rows, gate rows and widths (host only)."""
import ctypes

import pytest


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dim", [1, 40, 512, 513, 1280, 4096, 4097, 6144, 8192])
def test_join_workspace_is_bounded(dim, dtype):
    import paper_2607_08754_amd._lib as L
    n = ctypes.c_size_t()
    for groups in (1, 2, 100, 255, 256, 257, 511, 4095, 4096, 4097, 65536, 1 << 20):
        for run in (1, 2, 3, 5, 100, 4096):
            d = L.Join(groups * run, dim, dtype, L.LAYER, L.JOIN_POST | L.JOIN_PRE, groups, 0, 0, 0, 1e-5, 1.0, 0.0, 0)
            assert L.lib().slorr_join_workspace(d, n) == 0
            assert 0 < n.value < 128 << 20, (groups, run, n.value)
