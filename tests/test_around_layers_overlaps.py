"""Outputs over what else a call of norms or adapters reads or writes: refused before any HIP call (no GPU needed)."""
import ctypes
import os

import pytest

from paper_1804_02941_amd import binding, build

WORKSPACE, UNSUPPORTED = 4, 5
F32, BF16, F16 = binding.DAB_F32, binding.DAB_BF16, binding.DAB_F16
p = ctypes.c_void_p(4096)              # never dereferenced


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.lib()


# an output of 5 rows over a base at `at`: (the base's type, its rows' distance, where the output begins, in columns and bytes)
def overlaps(cols, own):
    size = {F32: 4, BF16: 2, F16: 2}
    wide = [] if own == F32 else [(F32, cols, 0), (F32, cols, 16), (F32, cols, 5 * cols * 4 - 16), (F32, cols + 8, 0)]
    return wide + [(own, cols + 8, 0), (own, cols, 16), (own, cols, -16), (own, cols, 5 * cols * size[own] - 16)]


@pytest.mark.parametrize("own", [F32, BF16, F16])
def test_adapters_output_over_base(lib, own):
    """Another workgroup's rows of base would be written before they are read."""
    X, base = 1 << 20, 1 << 21
    for t, ld, by in overlaps(24, own):
        assert lib.dab_adapters(X, own, 40, p, p, p, p, 5, 40, 24, 2, 3, base, t, ld, base + by, p, None) == UNSUPPORTED, (t, ld, by)


@pytest.mark.parametrize("own", [F32, BF16, F16])
def test_adapters_gradient_over_base(lib, own):
    dY, X, base = 1 << 19, 1 << 20, 1 << 21
    need = lib.dab_adapters_gradient_workspace_bytes(5, 40, 24, 2, 3)

    def call(t, ld, dX, T=5):
        return lib.dab_adapters_gradient(dY, 24, X, own, 40, p, p, p, p, p, T, 40, 24, 2, 3, base, t, ld, dX, p, p, None, need, None)
    for t, ld, by in overlaps(40, own):
        assert call(t, ld, base + by) == UNSUPPORTED, (t, ld, by)
    # element by element, one row, right before and right behind it: the next check's error
    assert call(own, 40, base) == WORKSPACE and call(own, 48, base, T=1) == WORKSPACE and call(F32, 40, base + 5 * 40 * 4) == WORKSPACE
    assert call(F32, 40, base - 5 * 40 * {F32: 4}.get(own, 2)) == WORKSPACE


@pytest.mark.parametrize("own", [F32, BF16, F16])
def test_norm_output_over_its_sum(lib, own):
    """What the gradient takes as h would be the norm's output."""
    X, R, H = 1 << 19, 1 << 20, 1 << 21
    size = 5 * 40 * (4 if own == F32 else 2)

    def call(h, y, r=R):
        return lib.dab_rms_norm(X, own, 40, r, 40, p, 1e-5, 5, 40, h, y, p, p, p, None)
    for by in (0, 16, -16, size - 16, 16 - size):
        assert call(H, H + by) == UNSUPPORTED, by
    assert call(X, X) == UNSUPPORTED and call(R, R) == UNSUPPORTED          # each alone may be where it is
