"""Norms of rows that four vectors a lane hold, 64 to 1024 lanes a row: sizes past those whose rows are spread over as many lanes as they have vectors.

The bounds are those of the norm's other tests, output by output and rstd among them, which its gradients take as it is.
"""
import pytest
import torch

from paper_1804_02941_amd import binding as dab
from test_gpu_norm import TYPES, check_norm, inputs, strided

pytestmark = pytest.mark.gpu

# more than 2^20 elements each; columns of 64 lanes with two and four vectors, 128, 256, 512, 1024, and the longest that these hold
SIZES = [(2100, 512), (1100, 1003), (600, 2001), (513, 2048), (523, 2049), (300, 4096), (250, 5003), (129, 8192), (129, 16383), (70, 16392), (40, 32761), (33, 32768)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_norm(dtype, rows, cols):
    assert rows * cols > 1 << 20
    x, r, gain, _, _ = inputs(rows, cols, dtype, 4)
    check_norm(x, None, gain, 1e-5, dab.dab_rms_norm(x, gain, eps=1e-5))
    check_norm(x, r, gain, 1e-5, dab.dab_rms_norm(strided(x, 3, 0), gain, residual=strided(r, 5, 8), eps=1e-5, save=True))
    got = dab.dab_rms_norm(x, gain, residual=r, eps=1e-5, save="only")
    assert got[0] is None
    check_norm(x, r, gain, 1e-5, got)
    # the sum over the residual and the output over the input
    Y, H, rstd, _ = dab.dab_rms_norm(x, gain, residual=r, eps=1e-5)
    a, b = x.clone(), r.clone()
    again = dab.dab_rms_norm(a, gain, residual=b, eps=1e-5, out=(a, b, None, None))
    assert torch.equal(a, Y) and torch.equal(b, H) and torch.equal(again[2], rstd)
