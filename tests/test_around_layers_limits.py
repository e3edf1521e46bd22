"""A norm of more threads than a launch takes along a dimension is refused before any HIP call (no GPU needed)."""
import ctypes
import os

import pytest

from paper_1804_02941_amd import binding, build

UNSUPPORTED = 5
p = ctypes.c_void_p(4096)              # never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.lib()


@pytest.mark.parametrize("rows,cols", [(1 << 30, 8), (1 << 30, 32), (1 << 26, 2048), (1 << 24, 8192), (1 << 22, 32769)])
def test_norm(lib, rows, cols):
    assert lib.dab_rms_norm(1 << 20, binding.DAB_BF16, cols, None, 0, p, 1e-5, rows, cols, None, 1 << 50, None, None, p, None) == UNSUPPORTED
