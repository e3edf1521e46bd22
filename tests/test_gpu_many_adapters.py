"""As many adapters as a call takes, almost all of them without tokens."""
import pytest
import torch

from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,K,F", [(3, 16, 24), (400, 16, 24), (150, 200, 130), (90, 5, 40)])
def test_many_adapters(dtype, T, K, F):
    n, r = 65535, 2
    g = torch.Generator(device=DEV).manual_seed(T)
    X, dY, A, B = (torch.randint(-2, 3, s, generator=g, device=DEV).to(dtype) for s in ((T, K), (T, F), (n, r, K), (n, r, F)))
    scale = 2.0 ** torch.randint(-1, 2, (n,), generator=g, device=DEV)
    ids = torch.randint(0, n, (T,), generator=g, device=DEV)
    ids[:3] = torch.tensor([0, n - 1, n], device=DEV)               # the last one is none
    ids[T // 2:T // 2 + 40] = ids[T // 2]
    some = ids < n
    i = ids.clamp(max=n - 1)
    x, dy, a, b = X.double(), dY.double(), A.double(), B.double()
    s = torch.where(some, scale[i], torch.zeros_like(scale[i])).double()
    u = (a[i] * x[:, None, :]).sum(dim=2) * some[:, None]
    v = (b[i] * dy[:, None, :]).sum(dim=2) * s[:, None]
    Y, U = dab.dab_adapters(X, ids.int(), A, B, scale.float(), base=dY)
    assert torch.equal(U.double(), u) and torch.equal(Y, (dy + s[:, None] * (u[:, :, None] * b[i]).sum(dim=1)).to(dtype))
    dX, dA, dB = dab.dab_adapters_gradient(dY, X, U, ids.int(), A, B, scale.float(), base=X)
    assert torch.equal(dX, (x + (v[:, :, None] * a[i]).sum(dim=1)).to(dtype))
    for got, rows, long in ((dA, v, x), (dB, s[:, None] * u, dy)):
        want = torch.zeros(got.shape, dtype=torch.float64, device=DEV)
        for t in range(T):
            if bool(some[t]):
                want[i[t]] += rows[t][:, None] * long[t][None, :]
        assert torch.equal(got.double(), want)
