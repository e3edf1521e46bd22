"""Saved inputs, 4-bit weights and the head's loss through the C ABI, against float64 (oracle/real_ends.py).

Codes, scales and restored values are equal to the oracle's.  Products are compared in two ways: on small whole numbers,
where every sum is exact and outputs have to be equal, and on random values with an error that the arithmetic allows:
u = 2^-24 for an fp32 operation (counted once per term of a sum, the most that any order of summation rounds), 2^-8
for a value rounded to bf16, 2^-11 for f16 (half of the last of p bits, over the smallest number of p bits: 2^-p).
"""
import numpy as np
import pytest
import torch

from oracle import real_ends as oe
from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
PIECES = {torch.float32: 3, torch.bfloat16: 1, torch.float16: 2}


def on_gpu(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(DEV)


def f64(t):
    return t.double().cpu().numpy()


def strided(t, extra, lead):
    """The same matrix as columns lead .. of a wider one whose other columns are NaN."""
    rows, cols = t.shape
    wide = torch.full((rows, cols + extra + lead), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, lead:lead + cols] = t
    return wide[:, lead:lead + cols]


def activations(rng, rows, cols):
    x = rng.standard_normal((rows, cols)) * np.exp(rng.normal(size=(1, cols)))
    x[rng.random(rows) < 0.1] = 0
    return x


# ------------------------------------------------------------------ saved inputs
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 31), (2, 32), (5, 33), (17, 100), (64, 512), (9, 520), (33, 1000), (2, 4097), (301, 64)])
def test_save_and_restore(dtype, rows, cols):
    x = on_gpu(activations(np.random.default_rng(rows * 1000 + cols), rows, cols), dtype)
    Qo, So = oe.save8(f64(x))
    for X in (x, strided(x, 3, 0), strided(x, 8, 8)):
        Q, S = dab.dab_ckpt8_save(X)
        assert np.array_equal(Q.cpu().numpy(), Qo) and np.array_equal(S.cpu().numpy(), So)
    back = oe.restore8(Qo, So, cols)
    for out in TYPES:
        want = torch.from_numpy(back).to(out)
        assert torch.equal(dab.dab_ckpt8_restore(Q, S, cols, out).cpu(), want)
        wide = torch.full((rows, cols + 5), 7.0, dtype=out, device=DEV)
        dab.dab_ckpt8_restore(Q, S, cols, out=wide[:, :cols])
        assert torch.equal(wide[:, :cols].cpu(), want) and bool((wide[:, cols:] == 7).all())


def test_saved_extremes_ties_and_what_is_not_finite():
    x = np.zeros((1, 32 * 10), dtype=np.float32)
    g = x.reshape(10, 32)
    g[0, :3] = [3.4e38, -3.4e38, 1e38]                            # the largest exponent
    g[1, :3] = [1e-45, 2 ** -130, -(2 ** -126)]                   # subnormal: below the smallest step
    g[2, :3] = [2.0 ** -104, 2.0 ** -110, 2.0 ** -111]            # the smallest exponent, a whole step and half of one
    g[3, :5] = [64, 0.5, 1.5, 2.5, -0.5]                          # ties
    g[4, :2] = [127.5, 63.75]
    g[5, 7] = np.inf
    g[6, 31] = np.nan
    g[7, 0] = -np.inf
    g[9, :2] = [127.49999, -127.49999]
    Q, S = dab.dab_ckpt8_save(on_gpu(x, torch.float32))
    Qo, So = oe.save8(x)
    assert np.array_equal(Q.cpu().numpy(), Qo) and np.array_equal(S.cpu().numpy(), So)
    assert So[0, 5] == So[0, 6] == So[0, 7] == 255
    back = dab.dab_ckpt8_restore(Q, S, x.shape[1]).cpu().numpy()
    np.testing.assert_array_equal(back, oe.restore8(Qo, So, x.shape[1]).astype(np.float32))
    assert np.isnan(back.reshape(10, 32)[5:8]).all()


def test_save_of_a_slice_whose_offsets_pass_32_bits():
    rows, ld, cols = 70000, 32768, 40                              # 2.3e9 elements between the first and the last
    wide = torch.empty((rows, ld), dtype=torch.bfloat16, device=DEV)
    x = wide[:, 64:64 + cols]
    x.normal_()
    Q, S = dab.dab_ckpt8_save(x)
    back = dab.dab_ckpt8_restore(Q, S, cols, torch.bfloat16)
    ref = dab.dab_ckpt8_restore(*dab.dab_ckpt8_save(x.contiguous()), cols, torch.bfloat16)
    assert torch.equal(back, ref)
    tail = f64(x[-5:])
    assert np.array_equal(f64(back[-5:]), oe.restore8(*oe.save8(tail), cols))
    dab.dab_ckpt8_restore(Q, S, cols, out=wide[:, 128:128 + cols])
    assert torch.equal(wide[:, 128:128 + cols], ref)


# ------------------------------------------------------------------ the weight gradient from a saved input
GRADS = [(1, 1, 1), (1, 300, 5), (63, 32, 64), (64, 129, 128), (65, 100, 127), (200, 257, 300), (1000, 40, 9), (129, 1000, 260), (4096, 64, 32)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,F", GRADS)
def test_weight_gradient(dtype, rows, cols, F):
    rng = np.random.default_rng(rows + cols + F)
    # whole numbers: bytes of a group with 64 among them have step 1, so nothing is lost and every sum is exact
    x = rng.integers(-60, 61, (rows, cols)).astype(np.float64)
    x[:, ::32] = 64
    y = rng.integers(-3, 4, (rows, F)).astype(np.float64)
    Q, S = dab.dab_ckpt8_save(on_gpu(x, torch.float32))
    for dY in (on_gpu(y, dtype), strided(on_gpu(y, dtype), 3, 0), strided(on_gpu(y, dtype), 16, 8)):
        dW = dab.dab_ckpt8_weight_gradient(dY, Q, S, cols)
        assert dW.dtype == torch.float32 and np.array_equal(f64(dW), y.T @ x)
    # random values: every product is exact, the sum rounds once per term (and per piece)
    x = on_gpu(activations(rng, rows, cols), torch.bfloat16)
    dY = on_gpu(0.01 * rng.standard_normal((rows, F)), dtype)
    Q, S = dab.dab_ckpt8_save(x)
    xo, yo = oe.restore8(*oe.save8(f64(x)), cols), f64(dY)
    dW = f64(dab.dab_ckpt8_weight_gradient(dY, Q, S, cols))
    assert np.all(np.abs(dW - yo.T @ xo) <= (rows * PIECES[dtype] + 2) * U * (np.abs(yo).T @ np.abs(xo)) + 1e-30)


def test_weight_gradient_is_the_upstream_gradient_of_a_binarized_layer():
    """Differences: the loss sum(Y * R) of the weights-only layer changes with W~ as dW says (the layer is linear in W~)."""
    rng = np.random.default_rng(3)
    B, K, F = 48, 96, 20
    X = on_gpu(rng.standard_normal((B, K)), torch.float32)
    R = on_gpu(rng.standard_normal((B, F)), torch.float32)
    Q, S = dab.dab_ckpt8_save(X)
    Xr = f64(dab.dab_ckpt8_restore(Q, S, K))
    dW = f64(dab.dab_ckpt8_weight_gradient(R, Q, S, K))
    W = rng.standard_normal((F, K))
    d = rng.standard_normal((F, K))
    f = lambda w: float(np.sum((Xr @ w.T) * f64(R)))               # noqa: E731
    slope = (f(W + 0.5 * d) - f(W - 0.5 * d))
    assert abs(float(np.sum(dW * d)) - slope) <= (3 * B + 2) * U * float(np.sum((np.abs(f64(R)).T @ np.abs(Xr)) * np.abs(d))) + 1e-9 * abs(slope)


# ------------------------------------------------------------------ 4-bit weights
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("F,K", [(1, 1), (5, 31), (16, 128), (17, 129), (33, 512), (20, 640), (3, 1000), (100, 96)])
def test_pack_and_unpack(dtype, F, K):
    rng = np.random.default_rng(F * 100 + K)
    w = on_gpu(rng.standard_normal((F, K)) * np.exp(rng.normal(size=(F, 1))), dtype)
    w[F // 2] = 0
    codes, scale = oe.pack4(f64(w))
    Qo, So = oe.tiles4(codes, scale)
    for W in (w, strided(w, 3, 0), strided(w, 8, 16)):
        Q, S = dab.dab_w4_pack(W)
        assert np.array_equal(Q.cpu().numpy(), Qo) and np.array_equal(S.cpu().numpy(), So)
    assert np.array_equal(f64(dab.dab_w4_unpack(Q, S, F, K)), oe.value4(codes, scale, K))


def test_pack_extremes_ties_and_what_is_not_finite():
    w = np.zeros((2, 32 * 5), dtype=np.float32)
    g = w.reshape(10, 32)
    g[0, :11] = [0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.9, -0.0, -7.0]
    g[1, :3] = [7.01, 1.0, -3.0]
    g[2, :2] = [3e38, -2e37]
    g[3, :2] = [1e-45, 1e-38]
    g[4, :4] = [2.0 ** -108, 2.0 ** -110, 2.0 ** -111, 2.0 ** -112]
    g[5, 3], g[6, 30], g[8, 0] = np.inf, np.nan, -np.inf
    Q, S = dab.dab_w4_pack(on_gpu(w, torch.float32))
    codes, scale = oe.pack4(w)
    Qo, So = oe.tiles4(codes, scale)
    assert np.array_equal(Q.cpu().numpy(), Qo) and np.array_equal(S.cpu().numpy(), So)
    back = dab.dab_w4_unpack(Q, S, 2, 160).cpu().numpy()
    np.testing.assert_array_equal(back, oe.value4(codes, scale, 160).astype(np.float32))
    X = torch.ones((1, 160), dtype=torch.bfloat16, device=DEV)
    Y = dab.dab_w4_matvec(X, Q, S, 2)
    assert not bool(torch.isfinite(Y[0, 1]))                      # its weights are not finite either


MATVECS = [(1, 1, 1), (1, 8, 16), (1, 4096, 33), (2, 130, 17), (3, 1000, 100), (5, 513, 40), (7, 96, 300), (8, 2048, 64), (16, 384, 48),
           (17, 136, 31), (22, 264, 20), (33, 128, 65), (64, 520, 16), (65, 72, 18), (200, 160, 35)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,K,F", MATVECS)
def test_matvec(dtype, B, K, F):
    rng = np.random.default_rng(B + K + F)
    # whole numbers and halves, exact in every type: sums below 2^24 halves come out exactly (16-bit outputs rounded once)
    levels = np.array(oe.LEVELS + tuple(-v for v in oe.LEVELS))
    w = levels[rng.integers(0, 16, (F, K))]
    w[:, ::32] = 6
    x = rng.integers(-4, 5, (B, K)).astype(np.float64)
    Q, S = dab.dab_w4_pack(on_gpu(w, torch.float32))
    want = torch.from_numpy(x @ w.T).to(dtype)
    for X in (on_gpu(x, dtype), strided(on_gpu(x, dtype), 3, 0), strided(on_gpu(x, dtype), 8, 8)):
        Y = dab.dab_w4_matvec(X, Q, S, F)
        assert Y.dtype == dtype and torch.equal(Y.cpu(), want)
    X = on_gpu(rng.standard_normal((B, K)), dtype)
    W = rng.standard_normal((F, K)) / np.sqrt(K)
    wo, xo = oe.value4(*oe.pack4(W.astype(np.float32)), K), f64(X)
    Q, S = dab.dab_w4_pack(on_gpu(W, torch.float32))
    ref = xo @ wo.T
    err = np.abs(f64(dab.dab_w4_matvec(X, Q, S, F)) - ref)
    assert np.all(err <= (PIECES[dtype] * K + 8) * U * (np.abs(xo) @ np.abs(wo).T) * (1 + HALF[dtype]) + HALF[dtype] * np.abs(ref) + 2.0 ** -25)


def test_matvec_with_more_codes_than_32_bits_reach():
    F, K = 131072 * 4, 16384                                       # 4.3e9 bytes of codes
    Q = torch.randint(0, 256, (F // 16, K // 128, 64, 16), dtype=torch.uint8, device=DEV)
    S = torch.full((F // 16, K // 512, 64, 4), 120, dtype=torch.uint8, device=DEV)
    X = torch.randint(-2, 3, (1, K), device=DEV).bfloat16()
    Y = dab.dab_w4_matvec(X.float(), Q, S, F)
    few = slice(F // 16 - 2, F // 16)
    W = dab.dab_w4_unpack(Q[few].contiguous(), S[few].contiguous(), 32, K)
    assert torch.equal(Y[0, -32:].double(), (W.double() @ X[0].double()))


# ------------------------------------------------------------------ the head
HEADS = [(1, 1, 1), (1, 64, 1000), (2, 8, 3), (7, 33, 50), (33, 64, 257), (64, 100, 300), (130, 72, 515), (5, 200, 4100), (300, 40, 129)]


def head_case(rng, T, D, V, dtype, ignored):
    H, W = on_gpu(rng.standard_normal((T, D)), dtype), on_gpu(2.0 / np.sqrt(D) * rng.standard_normal((V, D)), dtype)
    t = rng.integers(0, V, T)
    t[rng.random(T) < ignored] = -100
    return H, W, t, rng.random(T) + 0.5


def check_head(H, W, t, g, ignore=-100):
    """Loss and gradients against the oracle, with the errors that the arithmetic allows."""
    T, D = H.shape
    V, dtype = W.shape[0], H.dtype
    targets = torch.from_numpy(t).to(DEV)
    G = torch.from_numpy(g.astype(np.float32)).to(DEV)
    loss, lse = dab.dab_head_loss(H, W, targets, ignore_index=ignore)
    dH, dW = dab.dab_head_loss_gradient(H, W, targets, lse, G, ignore_index=ignore)
    h, w = np.nan_to_num(f64(H), nan=0.0, posinf=0.0, neginf=0.0), f64(W)
    o_loss, o_lse, P, o_dH, o_dW = oe.head(h, w, t, f64(G), ignore)
    live = (t != ignore) & (t >= 0) & (t < V)
    # a logit rounds once per term and piece pair; exp and log add a few last bits of fp32
    pairs = 6 if dtype == torch.float32 else 1
    logit = (pairs * D + 4) * U * (np.abs(h) @ np.abs(w).T).max(axis=1, initial=0)
    tol = 2 * logit + (V / 64 + 64) * U + 4 * U * np.abs(o_lse)
    assert np.all(np.abs(f64(loss) - o_loss)[live] <= tol[live]) and np.all(np.abs(f64(lse) - o_lse)[live] <= tol[live])
    assert not f64(loss)[t == ignore].any()
    # an entry of P: off by the logit's and lse's error, and rounded to bf16 where the inputs are bf16
    dP = np.abs(P) * (HALF[dtype] if dtype == torch.bfloat16 else 4 * U) + np.abs(g)[:, None] * live[:, None] * np.exp(np.minimum(h @ w.T - o_lse[:, None], 0)) * (tol + logit + 64 * U)[:, None] * 2
    for got, ref, err, terms in ((dH, o_dH, dP @ np.abs(w), V), (dW, o_dW, dP.T @ np.abs(h), T)):
        mag = (np.abs(P) @ np.abs(w)) if terms == V else (np.abs(P).T @ np.abs(h))
        allowed = err + (pairs * terms + 4) * U * mag + HALF[dtype] * np.abs(ref)
        assert np.all(np.abs(f64(got) - ref) <= 1.02 * allowed + 1e-30)
        # and, over the whole of it, what roundings of that size amount to
        assert np.linalg.norm(f64(got) - ref) <= (4e-3 if dtype == torch.bfloat16 else 2e-6 * max(1.0, np.abs(h @ w.T).max())) * np.linalg.norm(ref) + 1e-30
    assert not f64(dH)[~live].any()
    return loss, lse, dH, dW


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,D,V", HEADS)
def test_head(dtype, T, D, V):
    rng = np.random.default_rng(T + D + V)
    check_head(*head_case(rng, T, D, V, dtype, 0.3))


# sizes past what the kernels for small heads take (1024 or, in fp32, 4096 of anything), odd ones among them
TILED = [(1, 64, 5000), (2, 8, 4099), (7, 33, 4500), (33, 64, 4257), (64, 100, 5300), (130, 72, 4615), (300, 40, 4129), (4097, 24, 40), (100, 4200, 33),
         (1, 1, 4097), (129, 129, 4233)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,D,V", TILED)
def test_head_on_tiles(dtype, T, D, V):
    rng = np.random.default_rng(T + D + V)
    H, W, t, g = head_case(rng, T, D, V, dtype, 0.3)
    want = check_head(H, W, t, g)
    got = check_head(strided(H, 5, 0), strided(W, 8, 8), t, g)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_head_on_tiles_ignored_tokens_hold_anything():
    rng = np.random.default_rng(2)
    H, W, t, g = head_case(rng, 300, 48, 4400, torch.bfloat16, 0.0)
    t[5:9], t[20], t[280:] = -100, -100, -100
    t[1], t[2] = 4400, -1
    H[5], H[6], H[7, 3], H[20], H[299] = float("nan"), float("inf"), float("-inf"), float("nan"), float("inf")
    loss, lse, dH, dW = check_head(H, W, t, g)
    assert bool(torch.isfinite(dH).all()) and bool(torch.isfinite(dW).all()) and bool(torch.isnan(loss[1:3]).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_head_of_many_tiles_and_pieces(dtype):
    """Large tiles, several shares; a second run gives the same bits."""
    rng = np.random.default_rng(11)
    H, W, t, g = head_case(rng, 2000, 136, 7001, dtype, 0.2)
    first = check_head(H, W, t, g)
    again = check_head(H, W, t, g)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_head_in_several_pieces_of_the_vocabulary():
    """More words than one piece holds: against the same loss in float32 on the GPU."""
    T, D, V = 4096, 64, 70001
    g = torch.Generator(device=DEV).manual_seed(4)
    H = torch.randn((T, D), generator=g, device=DEV).bfloat16()
    W = (0.3 * torch.randn((V, D), generator=g, device=DEV)).bfloat16()
    t = torch.randint(0, V, (T,), generator=g, device=DEV)
    t[::7] = -100
    assert dab.lib().dab_head_loss_gradient_workspace_bytes(T, D, V, dab.DAB_BF16, D, D) < 2 * T * V
    loss, lse = dab.dab_head_loss(H, W, t)
    dH, dW = dab.dab_head_loss_gradient(H, W, t, lse)
    live = (t != -100).unsqueeze(1)
    L = torch.where(live, H.float(), 0.0) @ W.float().t()
    ref = torch.logsumexp(L, 1)
    assert torch.allclose(lse, torch.where(live[:, 0], ref, 0.0), rtol=1e-5, atol=1e-5)
    P = torch.exp(L - ref[:, None])
    P[torch.arange(T, device=DEV), t.clamp(min=0)] -= 1
    P = torch.where(live, P, 0.0)
    for got, want in ((dH, P @ W.float()), (dW, P.t().contiguous() @ torch.where(live, H.float(), 0.0))):
        assert float((got.float() - want).norm() / want.norm()) < 4e-3


def test_head_ignored_tokens_hold_anything():
    rng = np.random.default_rng(2)
    H, W, t, g = head_case(rng, 40, 48, 200, torch.bfloat16, 0.0)
    t[5:9], t[20] = -100, -100
    H[5], H[6], H[7, 3], H[20] = float("nan"), float("inf"), float("-inf"), float("nan")
    g[5] = np.nan
    check_head(H, W, t, np.where(np.isnan(g), 1.0, g))
    loss, lse = dab.dab_head_loss(H, W, torch.from_numpy(t).to(DEV))
    dH, dW = dab.dab_head_loss_gradient(H, W, torch.from_numpy(t).to(DEV), lse, torch.from_numpy(g.astype(np.float32)).to(DEV))
    assert bool(torch.isfinite(dH).all()) and bool(torch.isfinite(dW).all()) and not bool(loss[5].any()) and not bool(lse[5].any())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_head_without_any_token(dtype):
    rng = np.random.default_rng(2)
    H, W, t, g = head_case(rng, 33, 24, 90, dtype, 1.1)
    loss, lse, dH, dW = check_head(H, W, t, g)
    assert not any(bool(x.any()) for x in (loss, lse, dH, dW))


def test_head_targets_outside_the_vocabulary():
    rng = np.random.default_rng(2)
    H, W, t, g = head_case(rng, 12, 24, 90, torch.bfloat16, 0.0)
    t[1], t[2], t[3], t[4] = 90, -1, 2 ** 40, 7
    loss, lse, dH, dW = check_head(H, W, t, g, ignore=7)
    assert bool(torch.isnan(loss[1:4]).all()) and float(loss[4]) == 0


def test_head_of_large_logits_and_equal_ones():
    """Logits of hundreds (their exponentials leave fp32's range), and a row where every word is as likely."""
    rng = np.random.default_rng(2)
    H, W, t, g = head_case(rng, 20, 32, 333, torch.float32, 0.0)
    H[:8] *= 100
    H[9] = 0
    loss, lse, *_ = check_head(H, W, t, g)
    assert float(lse[9]) == pytest.approx(np.log(333), abs=1e-6)


def test_head_gradient_against_differences():
    """The change of the loss itself, fp32, along a random direction of H and of W.  With logits of a few units the
    difference quotient's own error is that of the loss, a few u |loss|, over the step, and the step squared."""
    rng = np.random.default_rng(8)
    T, D, V, eps = 60, 40, 300, 2.0 ** -8
    H, W, t, g = head_case(rng, T, D, V, torch.float32, 0.2)
    targets, G = torch.from_numpy(t).to(DEV), torch.from_numpy(g.astype(np.float32)).to(DEV)
    loss, lse = dab.dab_head_loss(H, W, targets)
    dH, dW = dab.dab_head_loss_gradient(H, W, targets, lse, G)
    for X, dX in ((H, dH), (W, dW)):
        d = on_gpu(rng.standard_normal(X.shape) / np.sqrt(D), torch.float32)
        at = []
        for s in (eps, -eps):
            args = (X + s * d, W) if X is H else (H, X + s * d)
            at.append(float((dab.dab_head_loss(*args, targets)[0].double() * G.double()).sum()))
        slope = (at[0] - at[1]) / (2 * eps)
        want = float((dX.double() * d.double()).sum())
        noise = float((loss.double() * G.double()).sum()) * 64 * U / eps
        assert abs(slope - want) <= noise + T * 4 * eps ** 2


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_head_of_strided_matrices(dtype):
    rng = np.random.default_rng(4)
    H, W, t, g = head_case(rng, 70, 56, 140, dtype, 0.2)
    want = check_head(H, W, t, g)
    for extra, lead in ((3, 0), (8, 8), (40, 16)):
        got = check_head(strided(H, extra, lead), strided(W, extra, lead), t, g)
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_head_of_a_matrix_whose_offsets_pass_32_bits():
    T, D, V = 3, 8192, 270000                                      # 2.2e9 weights
    W = torch.empty((V, D), dtype=torch.bfloat16, device=DEV).normal_(0, 0.02)
    H = torch.randn((T, D), device=DEV).bfloat16()
    t = torch.tensor([V - 1, 5, V - 2], device=DEV)
    loss, lse = dab.dab_head_loss(H, W, t)
    dH, dW = dab.dab_head_loss_gradient(H, W, t, lse)
    L = torch.cat([H.float() @ W[i:i + 30000].float().t() for i in range(0, V, 30000)], 1)
    assert torch.allclose(loss, torch.logsumexp(L, 1) - L.gather(1, t[:, None])[:, 0], rtol=1e-5)
    P = torch.softmax(L, 1)
    P.scatter_add_(1, t[:, None], torch.full((T, 1), -1.0, device=DEV))
    want = P[:, -40:].t().contiguous() @ H.float()
    assert float((dW[-40:].float() - want).norm() / want.norm()) < 4e-3
    want = sum(P[:, i:i + 30000] @ W[i:i + 30000].float() for i in range(0, V, 30000))
    assert float((dH.float() - want).norm() / want.norm()) < 4e-3


@pytest.mark.parametrize("rows,cols,F", [(20000, 40, 70), (1030, 520, 300), (512, 2600, 1300), (257, 4100, 4100), (6000, 260, 516)])
@pytest.mark.parametrize("dtype", TYPES)
def test_weight_gradient_of_shared_and_whole_tiles(dtype, rows, cols, F):
    """Rounds of whole tiles, a last round in shares, long sums of few tiles: whole numbers, equal."""
    rng = np.random.default_rng(rows)
    x = rng.integers(-15, 16, (rows, cols)).astype(np.float64)
    x[:, ::32] = 64
    y = rng.integers(-3, 4, (rows, F)).astype(np.float64)
    Q, S = dab.dab_ckpt8_save(on_gpu(x, torch.bfloat16))
    dW = dab.dab_ckpt8_weight_gradient(on_gpu(y, dtype), Q, S, cols)
    assert torch.equal(dW.double(), torch.mm(on_gpu(y, torch.float64).t().contiguous(), on_gpu(x, torch.float64)))


# ------------------------------------------------------------------ streams, graphs, refusals
def test_calls_go_to_the_current_stream_and_into_a_graph():
    rng = np.random.default_rng(6)
    H, W, t, g = head_case(rng, 100, 64, 300, torch.bfloat16, 0.2)
    targets = torch.from_numpy(t).to(DEV)
    X = on_gpu(rng.standard_normal((100, 64)), torch.float32)
    Q4, S4 = dab.dab_w4_pack(W)

    def step():
        loss, lse = dab.dab_head_loss(H, W, targets)
        dH, dW = dab.dab_head_loss_gradient(H, W, targets, lse)
        Q, S = dab.dab_ckpt8_save(X)
        return loss, dH, dW, dab.dab_ckpt8_weight_gradient(dH, Q, S, 64), dab.dab_w4_matvec(X, Q4, S4, 300)

    want = [a.clone() for a in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    for _ in range(4):
        for a in got:
            a.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        eager = step()
        assert all(torch.equal(a, b) for a, b in zip(eager, want))


def test_refusals_of_the_binding():
    X = torch.randn((4, 64), device=DEV)
    Q, S = dab.dab_ckpt8_save(X)
    with pytest.raises(TypeError, match="X: expected torch.float32, torch.bfloat16 or torch.float16"):
        dab.dab_ckpt8_save(X.double())
    with pytest.raises(TypeError, match="tensor on the GPU"):
        dab.dab_ckpt8_save(X.cpu())
    with pytest.raises(ValueError, match="contiguous"):
        dab.dab_ckpt8_save(X.t())
    with pytest.raises(ValueError, match="two dimensions"):
        dab.dab_ckpt8_save(X[0])
    with pytest.raises(ValueError, match="rows apart"):
        dab.dab_ckpt8_save(X[:1].expand(4, 64))
    with pytest.raises(dab.DabError, match="dab_ckpt8_save failed: status"):
        dab.dab_ckpt8_save(X[:0])
    with pytest.raises(dab.DabError, match="status 3"):
        dab.dab_ckpt8_save(X[:, 1:33])
    with pytest.raises(ValueError, match="Q: expected shape"):
        dab.dab_ckpt8_restore(Q, S, 65)
    with pytest.raises(ValueError, match="dY: expected shape"):
        dab.dab_ckpt8_weight_gradient(X[:3], Q, S, 64)
    with pytest.raises(TypeError, match="W: expected torch.float32"):
        dab.dab_head_loss(X, X.bfloat16(), torch.zeros(4, dtype=torch.int64, device=DEV))
    with pytest.raises(TypeError, match="targets: expected torch.int64"):
        dab.dab_head_loss(X, X, torch.zeros(4, dtype=torch.int32, device=DEV))
    with pytest.raises(dab.DabError, match="status 5"):
        dab.dab_head_loss(X.half(), X.half(), torch.zeros(4, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError, match="W: expected shape"):
        dab.dab_head_loss(X, X[:, :32], torch.zeros(4, dtype=torch.int64, device=DEV))
    Q4, S4 = dab.dab_w4_pack(X)
    with pytest.raises(ValueError, match="Q: expected shape"):
        dab.dab_w4_matvec(torch.randn((1, 200), device=DEV), Q4, S4, 4)
    with pytest.raises(ValueError, match="out: expected shape"):
        dab.dab_w4_matvec(X, Q4, S4, 4, out=torch.empty((4, 5), device=DEV))


# few tokens or few words beside a width past 4096, and sizes on either side of where the products change their tiles
@pytest.mark.parametrize("T,D,V", [(100, 4200, 17), (40, 4200, 32), (17, 4100, 1), (31, 4104, 300), (97, 500, 2600), (1025, 60, 1030), (300, 1504, 628), (520, 33, 9000)])
def test_fp32_head_on_every_tile(T, D, V):
    rng = np.random.default_rng(T + D + V)
    H, W, t, g = head_case(rng, T, D, V, torch.float32, 0.2)
    want = check_head(H, W, t, g)
    got = check_head(strided(H, 3, 0), strided(W, 4, 4), t, g)
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,D", [(1, 40), (100, 8), (189, 4534), (1094, 8), (4100, 24)])
def test_head_of_one_word_has_nothing_to_learn(dtype, T, D):
    rng = np.random.default_rng(T + D)
    loss, _, dH, dW = check_head(*head_case(rng, T, D, 1, dtype, 0.2))
    assert not loss.any() and not dH.any() and not dW.any()        # p = exp(0) exactly


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1, 40, 150, 1100])
@pytest.mark.parametrize("D", [1, 2, 33, 34, 38, 66, 100, 191])
def test_head_between_whatever_lies_behind_its_rows(dtype, T, D):
    """Rows of any number of words, each followed by what is no number: none of it is multiplied."""
    rng = np.random.default_rng(T + D)
    V = 4101
    H, W, t, g = head_case(rng, T, D, V, dtype, 0.1)
    want = check_head(H, W, t, g)
    for behind in (1, 2, 8 - D % 8):
        wide = torch.full((V, D + behind), float("nan"), dtype=dtype, device=DEV)
        wide[:, :D] = W
        last = torch.full((T, D + behind), float("inf"), dtype=dtype, device=DEV)
        last[:, :D] = H
        got = check_head(last[:, :D], wide[:, :D], t, g)
        assert all(torch.equal(a, b) for a, b in zip(want, got))
