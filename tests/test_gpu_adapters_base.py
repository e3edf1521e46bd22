"""Adapters whose output shares memory with base: in place for one row of any distance, refused where rows would be written before they are read."""
import pytest
import torch

from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T", [1, 5, 300])
def test_output_over_base(dtype, T):
    g = torch.Generator(device=DEV).manual_seed(T)
    K, F, n, r = 40, 24, 2, 3
    X, dY, A, B = (torch.randint(-2, 3, s, generator=g, device=DEV).to(dtype) for s in ((T, K), (T, F), (n, r, K), (n, r, F)))
    ids = torch.randint(-1, n, (T,), generator=g, device=DEV).int()
    Y, U = dab.dab_adapters(X, ids, A, B, base=dY)
    dX, dA, dB = dab.dab_adapters_gradient(dY, X, U, ids, A, B, base=X)
    calls = ((dY, Y, lambda base, out: dab.dab_adapters(X, ids, A, B, base=base, out=(out, None))[0]),
             (X, dX, lambda base, out: dab.dab_adapters_gradient(dY, X, U, ids, A, B, base=base, out=(out, None, None))[0]))
    for base, want, call in calls:
        cols = base.shape[1]
        wide = torch.zeros(T * (cols + 8), dtype=dtype, device=DEV)
        apart, first = wide.view(T, cols + 8)[:, :cols], wide[:T * cols].view(T, cols)
        apart.copy_(base)
        if T == 1:
            assert torch.equal(call(apart, first), want)
        else:
            with pytest.raises(dab.DabError, match="status 5"):
                call(apart, first)
            assert torch.equal(apart, base)                         # nothing was written
        if dtype != torch.float32:
            both = base.float()
            with pytest.raises(dab.DabError, match="status 5"):
                call(both, both.view(dtype).view(-1)[:T * cols].view(T, cols))
            assert torch.equal(both, base.float())
        assert torch.equal(call(base.clone(), None), want)
