"""A norm's sum and its output are two tensors: in each other's place they are refused, in the inputs' places they are kept apart."""
import pytest
import torch

from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,cols", [(1, 40), (5, 100), (3, 40000)])
def test_sum_and_output(dtype, rows, cols):
    g = torch.Generator(device=DEV).manual_seed(cols)
    x, r = (torch.randn((rows, cols), generator=g, device=DEV).to(dtype) for _ in range(2))
    gain = 1 + 0.1 * torch.randn(cols, generator=g, device=DEV)
    Y, H, _, _ = dab.dab_rms_norm(x, gain, residual=r)
    both, a, b = torch.zeros_like(x), x.clone(), r.clone()
    for out in (both, a, b):
        with pytest.raises(dab.DabError, match="status 5"):
            dab.dab_rms_norm(a, gain, residual=b, out=(out, out, None, None))
    assert not both.any() and torch.equal(a, x) and torch.equal(b, r)
    for out in ((a, b), (b, a)):
        a.copy_(x), b.copy_(r)
        dab.dab_rms_norm(a, gain, residual=b, out=(*out, None, None))
        assert torch.equal(out[0], Y) and torch.equal(out[1], H)
    # without a residual there is no sum to keep
    a.copy_(x)
    got = dab.dab_rms_norm(a, gain, out=(a, None, None, None))
    assert got[1] is a and torch.equal(a, dab.dab_rms_norm(x, gain)[0])
