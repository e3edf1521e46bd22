"""Adapters behind the 4-bit product at sizes that take its other forms: several tiles and groups a wavefront, up to eight shares of a row, several passes over the
tokens, adapters' rows read ahead of the product or behind it, and rows of U longer than a workgroup's first turn.

Whole and half numbers: every product and sum is exact in fp32 (below 2^22 in steps of a quarter), so outputs equal the definition's, rounded once.
"""
import pytest
import torch

from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# tokens, K, F, ranks
SIZES = [(1, 4096, 4099, (5, 70)),             # eight shares of a row, rows of the rank in one turn of eight lanes and in several
         (1, 520, 16400, (16,)),               # two tiles a wavefront, two groups
         (1, 512, 70000, (17,)),               # one share, eight groups
         (3, 4104, 16395, (24,)), (3, 1000, 33000, (5,)),
         (5, 9000, 520, (9,)),                 # more than 8192 k
         (7, 9111, 4099, (24,)),
         (17, 4200, 2061, (64,)),              # two columns of tokens or three, two passes in fp32
         (20, 300, 40000, (5, 24)),            # four tiles a wavefront, several groups, adapters behind the product
         (32, 700, 16395, (5, 24, 64, 256)), (32, 2000, 16395, (33,)),
         (48, 600, 8200, (8,)), (48, 4100, 8203, (24,)),
         (70, 4500, 16387, (7, 64)),           # U in a launch of its own
         # rows of fewer than eight
         (1, 40, 1, (1, 12)), (2, 64, 5, (3,)), (3, 5, 20, (4, 33)), (65, 130, 7, (20,)), (66, 7, 3, (2,))]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,K,F,ranks", SIZES)
def test_whole_numbers(dtype, T, K, F, ranks):
    g = torch.Generator(device=DEV).manual_seed(T + K + F)

    def whole(low, high, *shape):
        return torch.randint(low, high + 1, shape, generator=g, device=DEV).double()
    levels = torch.tensor([-6.0, -4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEV)
    W = levels[torch.randint(0, 15, (F, K), generator=g, device=DEV)]
    W[:, ::32] = 6                                                  # a group's largest: its scale is 1
    Q, S = dab.dab_w4_pack(W)
    X = whole(-2, 2, T, K)
    product = X @ W.double().t().contiguous()
    n = 3
    scale = 2.0 ** whole(-1, 1, n)
    for r in ranks:
        A, B = whole(-2, 2, n, r, K), whole(-2, 2, n, r, F)
        a, b, s = A.to(dtype), B.to(dtype), scale.float()
        some = torch.randint(-1, n, (T,), generator=g, device=DEV)
        for ids in (some, torch.full_like(some, n - 1), torch.full_like(some, n)):
            want = product.clone()
            for i in range(n):
                at = torch.nonzero(ids == i).squeeze(1)
                u = X[at] @ A[i].t().contiguous()
                want[at] += scale[i] * (u @ B[i])
            Y = dab.dab_w4_adapters(X.to(dtype), Q, S, F, ids.int(), a, b, s)
            assert float(want.abs().max()) < 2.0 ** 22 and torch.equal(Y, want.to(dtype)), r
        gap = torch.full((T, K + 3), float("nan"), dtype=dtype, device=DEV)       # rows that are not aligned
        gap[:, :K] = X.to(dtype)
        assert torch.equal(dab.dab_w4_adapters(gap[:, :K], Q, S, F, ids.int(), a, b, s), want.to(dtype))
