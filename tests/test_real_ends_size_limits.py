"""Sizes at the ends of what 32-bit counts hold: refused before anything is planned (no GPU needed; nothing here reaches a launch)."""
import ctypes
import os

import pytest

from paper_1804_02941_amd import binding, build

UNSUPPORTED = 5
p = ctypes.c_void_p(4096)              # never dereferenced
LAST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.lib()


@pytest.mark.parametrize("dtype", [binding.DAB_F32, binding.DAB_BF16, binding.DAB_F16])
@pytest.mark.parametrize("rows", [LAST, LAST - 1, LAST - 62])
def test_weight_gradient_of_more_rows_than_its_steps_count(lib, rows, dtype):
    """Steps of 64 rows are rounded up: the sum passes 2^31 from 2^31 - 63 rows on, and fewer steps than none are no sum."""
    assert lib.dab_ckpt8_weight_gradient_workspace_bytes(rows, 1, 1, dtype, 1) == 0
    assert lib.dab_ckpt8_weight_gradient(p, dtype, 1, p, p, rows, 1, 1, p, p, 2 ** 62, None) == UNSUPPORTED


def test_weight_gradient_of_as_many_rows_as_its_steps_count_is_planned(lib):
    rows = LAST - 63
    # the saved input and dY as bf16 (8 columns of it: 16-byte pieces)
    assert lib.dab_ckpt8_weight_gradient_workspace_bytes(rows, 1, 1, binding.DAB_BF16, 1) >= rows * (32 + 8) * 2
