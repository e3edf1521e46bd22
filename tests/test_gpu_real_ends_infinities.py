"""Infinities, NaN and the largest numbers in tokens and gradients, which the products take as sums of bf16 numbers: what comes out is what the
definition gives, an infinity of the same sign, NaN where one meets a zero or another, and numbers up to fp32's last."""
import numpy as np
import pytest
import torch

from oracle import real_ends as oe
from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LARGE = {torch.float32: 3.4028234e38, torch.bfloat16: 3.3895314e38, torch.float16: 65504.0}


def spoil(x, dtype):
    """Rows of x with something special each; the rest as they are."""
    x[0, 1] = np.inf
    x[1, 0] = -np.inf
    x[2, 2], x[2, 5] = np.inf, -np.inf
    x[3, 4] = np.nan
    x[4] = 0
    x[4, 3] = LARGE[dtype]
    x[5] = 0
    x[5, 6] = -LARGE[dtype]
    return x


def check(got, a, b, dtype, pieces):
    """got = a b^T, a with special values: term by term in float64."""
    with np.errstate(invalid="ignore", over="ignore"):
        terms = a[:, None, :] * b[None, :, :]
        want = terms.sum(axis=2)
        size = np.abs(np.where(np.isfinite(terms), terms, 0)).sum(axis=2)
    got = got.double().cpu().numpy()
    most = {torch.float32: 3.4028235e38, torch.bfloat16: 3.3895314e38, torch.float16: 65504.0}[dtype]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    infinite = np.isinf(want)
    assert np.array_equal(got[infinite], want[infinite])
    finite = np.isfinite(want)
    assert np.all(np.abs(want[finite]) < most)                     # (no overflow of the result's own among these inputs)
    limit = (pieces * a.shape[1] + 8) * 2.0 ** -24 * size + HALF[dtype] * np.abs(want) + 2.0 ** -25
    assert np.all(np.abs(got[finite] - want[finite]) <= limit[finite])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,K,F", [(6, 64, 40), (7, 130, 17), (20, 1000, 33)])
def test_4_bit_products(dtype, B, K, F):
    rng = np.random.default_rng(B + K)
    W = rng.choice([0.0, 0.5, -0.5, 0.25, -0.125, 0.75], (F, K))
    W[:, :8] = rng.choice([0.0, 0.5, -0.5, 0.25], (F, 8))
    Q, S = dab.dab_w4_pack(torch.from_numpy(W).float().to(DEV))
    assert np.array_equal(oe.value4(*oe.pack4(W), K), W)
    X = torch.from_numpy(spoil(rng.standard_normal((B, K)), dtype)).to(dtype)
    Y = dab.dab_w4_matvec(X.to(DEV), Q, S, F)
    check(Y, X.double().numpy(), W, dtype, {torch.float32: 3, torch.bfloat16: 1, torch.float16: 2}[dtype])
    for b in range(6):                                             # (a token by itself, which takes other kernels)
        y = dab.dab_w4_matvec(X[b:b + 1].clone().to(DEV), Q, S, F)
        check(y, X[b:b + 1].double().numpy(), W, dtype, 3)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,F", [(64, 40, 8), (300, 130, 17), (2000, 33, 70)])
def test_weight_gradient(dtype, rows, cols, F):
    rng = np.random.default_rng(rows)
    x = rng.integers(-32, 33, (rows, cols)) / 64.0
    x[:, ::32] = 1.0                                               # (steps of 1/64: nothing is lost)
    Q, S = dab.dab_ckpt8_save(torch.from_numpy(x).float().to(DEV))
    dY = torch.from_numpy(spoil(0.01 * rng.standard_normal((F, rows)), dtype).T.copy()).to(dtype)
    dW = dab.dab_ckpt8_weight_gradient(dY.to(DEV), Q, S, cols)
    check(dW, dY.double().numpy().T, x.T, torch.float32, {torch.float32: 3, torch.bfloat16: 1, torch.float16: 2}[dtype])


@pytest.mark.parametrize("T,D,V", [(3, 40, 300), (2100, 1024, 4225)])
def test_head_of_the_largest_numbers(T, D, V):
    """A token's largest number meets one small weight of each word, in the small kernels and as pieces."""
    g = torch.Generator(device=DEV).manual_seed(T)
    H, W = torch.zeros((T, D), device=DEV), torch.zeros((V, D), device=DEV)
    H[:, 5] = 3.4028234e38
    W[:, 5] = torch.randn((V,), generator=g, device=DEV) * 2.0 ** -127
    t = torch.randint(0, V, (T,), generator=g, device=DEV)
    loss, lse = dab.dab_head_loss(H, W, t)
    L = H[:1].double() @ W.double().t()
    assert float(L.abs().max()) < 20
    ref = torch.logsumexp(L, 1)
    # (weights below 2^-126 have fewer bits: pieces of them are whole steps of 2^-133, half of one off)
    tol = 1e-5 * 20 + float(2.0 ** -134 * H[0, 5].double())
    assert float((lse.double() - ref).abs().max()) <= tol and float((loss.double() - (ref - L[0, t])).abs().max()) <= 2 * tol
