"""Adapters beside a projection, their gradients, and with 4-bit weights, through the C ABI, against float64 (oracle/around_layers.py).

On small whole numbers every sum is exact, and outputs equal the definition's, rounded once to their type.  On random values the arithmetic allows an
error of u = 2^-24 for every fp32 operation, counted once per term of a sum (the most that any order rounds), and of half a step of
the output's type (bf16 2^-8, f16 2^-11 of the value).
"""
import numpy as np
import pytest
import torch

from oracle import around_layers as oa
from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
# tokens, K, F, adapters, rank: few and many tokens, every width of the rank, sizes that fit nothing
SIZES = [(1, 1, 1, 1, 1), (1, 40, 24, 3, 4), (3, 100, 130, 2, 16), (17, 64, 129, 5, 3), (33, 301, 70, 4, 8), (64, 129, 257, 7, 20), (65, 128, 128, 1, 16),
         (70, 33, 1000, 3, 17), (100, 257, 120, 2, 33), (130, 96, 260, 70, 5), (200, 520, 64, 4, 64), (257, 90, 40, 3, 70), (300, 40, 136, 2, 130), (1100, 64, 72, 3, 12),
         # rows of fewer than eight
         (100, 5, 40, 2, 3), (150, 40, 7, 3, 20), (90, 3, 2, 2, 4), (500, 8, 9, 2, 6)]


def f64(t):
    return t.double().cpu().numpy()


def on_gpu(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(DEV)


def strided(t, extra, lead):
    rows, cols = t.shape
    wide = torch.full((rows, cols + extra + lead), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, lead:lead + cols] = t
    return wide[:, lead:lead + cols]


def who(rng, T, n, form):
    if form == "runs":
        return np.repeat(rng.integers(-1, n, -(-T // 24)), 24)[:T].astype(np.int32)
    if form == "one":
        return np.full(T, n - 1, dtype=np.int32)
    if form == "none":
        return np.full(T, -1, dtype=np.int32)
    ids = rng.integers(0, n, T).astype(np.int32)                    # any order, and numbers that no adapter has
    ids[rng.random(T) < 0.2] = rng.choice([-1, n, 2 ** 31 - 1, -2 ** 31])
    return ids


def whole_numbers(rng, T, K, F, n, r):
    X, A, B, dY = (rng.integers(-2, 3, s).astype(float) for s in ((T, K), (n, r, K), (n, r, F), (T, F)))
    return X, A, B, dY, 2.0 ** rng.integers(-1, 2, n), rng.integers(-50, 51, (T, F)).astype(float), rng.integers(-50, 51, (T, K)).astype(float)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,K,F,n,r", SIZES)
def test_whole_numbers(dtype, T, K, F, n, r):
    rng = np.random.default_rng(T + K + F + n + r)
    X, A, B, dY, scale, base, dbase = whole_numbers(rng, T, K, F, n, r)
    x, a, b, dy, s = on_gpu(X, dtype), on_gpu(A, dtype), on_gpu(B, dtype), on_gpu(dY, dtype), on_gpu(scale, torch.float32)
    for form in ("runs", "any", "one", "none"):
        ids = who(rng, T, n, form)
        i = on_gpu(ids, torch.int32)
        Yo, Uo = oa.adapters(X, ids, A, B, scale, base)
        for bt in {dtype, torch.float32}:
            Y, got_u = dab.dab_adapters(strided(x, 3, 0), i, a, b, s, base=strided(on_gpu(base, bt), 1, 0))
            assert np.array_equal(f64(got_u), Uo) and torch.equal(Y, on_gpu(Yo, dtype))
        dXo, dAo, dBo = oa.adapters_gradient(dY, X, Uo, ids, A, B, scale, dbase)
        dX, dA, dB = dab.dab_adapters_gradient(strided(dy, 5, 0), strided(x, 1, 8), got_u, i, a, b, s, base=on_gpu(dbase, dtype))
        assert np.array_equal(f64(dA), dAo) and np.array_equal(f64(dB), dBo) and torch.equal(dX, on_gpu(dXo, dtype))
    # without a base, a scale and a gradient of the input
    Y, got_u = dab.dab_adapters(x, i, a, b)
    one = np.ones(n)
    Yo, Uo = oa.adapters(X, ids, A, B, one, None)
    assert torch.equal(Y, on_gpu(Yo, dtype))
    dX, dA, dB = dab.dab_adapters_gradient(dy, x, got_u, i, a, b, want_dX=False)
    _, dAo, dBo = oa.adapters_gradient(dY, X, Uo, ids, A, B, one, None)
    assert dX is None and np.array_equal(f64(dA), dAo) and np.array_equal(f64(dB), dBo)


def random_values(rng, T, K, F, n, r, dtype):
    X, A, B, dY = (on_gpu(k * rng.standard_normal(s), dtype) for s, k in (((T, K), 1), ((n, r, K), K ** -0.5), ((n, r, F), 0.3), ((T, F), 0.1)))
    return X, A, B, dY, on_gpu(0.5 + rng.random(n), torch.float32), on_gpu(rng.standard_normal((T, F)), dtype), on_gpu(0.1 * rng.standard_normal((T, K)), dtype)


def bounds(X, A, B, dY, scale, ids):
    """Sums of magnitudes: of U's, Y's, V's, dX's, dA's and dB's terms."""
    x, a, b, dy, s = (np.abs(f64(t)) for t in (X, A, B, dY, scale))
    n, r = a.shape[:2]
    Yb, Ub = oa.adapters(x, ids, a, b, s, None)
    dXb, dAb, dBb = oa.adapters_gradient(dy, x, Ub, ids, a, b, s, None)
    return Ub, Yb, dXb, dAb, dBb


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,K,F,n,r", SIZES)
def test_random_values(dtype, T, K, F, n, r):
    rng = np.random.default_rng(T + K + F + n + r + 1)
    X, A, B, dY, scale, base, dbase = random_values(rng, T, K, F, n, r, dtype)
    ids = who(rng, T, n, "runs")
    i = on_gpu(ids, torch.int32)
    Y, Ug = dab.dab_adapters(X, i, A, B, scale, base=base)
    Ub, Yb, dXb, dAb, dBb = bounds(X, A, B, dY, scale, ids)
    Yo, Uo = oa.adapters(f64(X), ids, f64(A), f64(B), f64(scale), f64(base))
    assert np.all(np.abs(f64(Ug) - Uo) <= (K + 1) * U * Ub)
    off = (K + r + 6) * U * Yb + U * np.abs(f64(base))
    assert np.all(np.abs(f64(Y) - Yo) <= off + HALF[dtype] * (np.abs(Yo) + off) + 2.0 ** -25 * (dtype == torch.float16))
    dX, dA, dB = dab.dab_adapters_gradient(dY, X, Ug, i, A, B, scale, base=dbase)
    dXo, dAo, dBo = oa.adapters_gradient(f64(dY), f64(X), Uo, ids, f64(A), f64(B), f64(scale), f64(dbase))
    off = (F + r + 6) * U * dXb + U * np.abs(f64(dbase))
    assert np.all(np.abs(f64(dX) - dXo) <= off + HALF[dtype] * (np.abs(dXo) + off) + 2.0 ** -25 * (dtype == torch.float16))
    assert np.all(np.abs(f64(dA) - dAo) <= (F + T + 6) * U * dAb) and np.all(np.abs(f64(dB) - dBo) <= (K + T + 6) * U * dBb)
    again = dab.dab_adapters_gradient(dY, X, Ug, i, A, B, scale, base=dbase)
    assert all(torch.equal(p, q) for p, q in zip(again, (dX, dA, dB)))


@pytest.mark.parametrize("dtype", TYPES)
def test_many_tokens(dtype):
    """More tokens than one share of the gradients' sums, long rows, an adapter that has none of the tokens."""
    rng = np.random.default_rng(5)
    T, K, F, n, r = 2500, 300, 260, 4, 16
    X, A, B, dY, scale, base, dbase = whole_numbers(rng, T, K, F, n, r)
    for ids in (np.repeat(rng.integers(0, 3, 50), 50).astype(np.int32), rng.integers(0, 3, T).astype(np.int32)):
        x, a, b, dy, s, i = on_gpu(X, dtype), on_gpu(A, dtype), on_gpu(B, dtype), on_gpu(dY, dtype), on_gpu(scale, torch.float32), on_gpu(ids, torch.int32)
        Y, Ug = dab.dab_adapters(x, i, a, b, s, base=on_gpu(base, torch.float32))
        Yo, Uo = oa.adapters(X, ids, A, B, scale, base)
        assert np.array_equal(f64(Ug), Uo) and torch.equal(Y, on_gpu(Yo, dtype))
        dX, dA, dB = dab.dab_adapters_gradient(dy, x, Ug, i, a, b, s)
        dXo, dAo, dBo = oa.adapters_gradient(dY, X, Uo, ids, A, B, scale, None)
        assert np.array_equal(f64(dA), dAo) and np.array_equal(f64(dB), dBo) and torch.equal(dX, on_gpu(dXo, dtype)) and not dA[3].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_share_of_more_tokens_than_lds_holds(dtype):
    """So many columns that the tokens are not shared out: 2500 of them a workgroup."""
    T, K, F, n, r = 2500, 16, 65600, 2, 3
    g = torch.Generator(device=DEV).manual_seed(4)
    X, dY, A, B = (torch.randint(-2, 3, s, generator=g, device=DEV).to(dtype) for s in ((T, K), (T, F), (n, r, K), (n, r, F)))
    ids = torch.randint(-1, n, (T,), generator=g, device=DEV).int()
    Y, Ug = dab.dab_adapters(X, ids, A, B)
    dX, dA, dB = dab.dab_adapters_gradient(dY, X, Ug, ids, A, B)
    for i in range(n):
        at = torch.nonzero(ids == i).squeeze(1)
        x, y, b = X[at].float(), dY[at].float(), B[i].float()
        u = x @ A[i].float().t()
        v = (y.double() @ b.double().t()).float()                  # whole numbers below 2^24: exact
        assert torch.equal(Ug[at], u) and torch.equal(dB[i], u.t().contiguous() @ y) and torch.equal(dA[i].double(), v.double().t().contiguous() @ x.double())
        assert torch.equal(dX[at], (v @ A[i].float()).to(dtype)) and torch.equal(Y[at], (u @ b).to(dtype))
    assert not dX[ids < 0].any()


@pytest.mark.parametrize("T", [3, 100, 400])
def test_the_smallest_f16_numbers_count(T):
    """Subnormal inputs, 2^-24 and its multiples, are not taken for zeros."""
    rng = np.random.default_rng(12)
    K, F, n, r = 96, 64, 2, 8
    X, A, B, dY, _, _, _ = whole_numbers(rng, T, K, F, n, r)
    ids = who(rng, T, n, "runs")
    x, a, b, dy, i = on_gpu(X * 2.0 ** -24, torch.float16), on_gpu(A, torch.float16), on_gpu(B, torch.float16), on_gpu(dY * 2.0 ** -24, torch.float16), on_gpu(ids, torch.int32)
    Y, Ug = dab.dab_adapters(x, i, a, b)
    Yo, Uo = oa.adapters(X, ids, A, B, np.ones(n), None)
    assert np.array_equal(f64(Ug), Uo * 2.0 ** -24) and torch.equal(Y, on_gpu(Yo * 2.0 ** -24, torch.float16))
    dX, dA, dB = dab.dab_adapters_gradient(dy, x, Ug, i, a, b)
    dXo, dAo, dBo = oa.adapters_gradient(dY, X, Uo, ids, A, B, np.ones(n), None)
    assert torch.equal(dX, on_gpu(dXo * 2.0 ** -24, torch.float16)) and np.array_equal(f64(dA), dAo * 2.0 ** -48) and np.array_equal(f64(dB), dBo * 2.0 ** -48)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("r", [5, 24, 64, 70])
@pytest.mark.parametrize("T,K,F,gap", [(200, 1337, 4099, 0), (200, 1337, 301, 6), (300, 600, 264, 1), (4200, 9, 1031, 4), (41, 771, 8, 1), (41, 7, 15, 2)])
def test_rows_at_odd_distances(dtype, r, T, K, F, gap):
    """16-bit rows every other one of which lies between two words; what is between the rows, NaN, does not get in."""
    rng = np.random.default_rng(T + K + F + r)
    n = 3
    X, A, B, dY, scale, base, dbase = whole_numbers(rng, T, K, F, n, r)
    a, b, s = on_gpu(A, dtype), on_gpu(B, dtype), on_gpu(scale, torch.float32)

    def apart(m):
        wide = torch.full((T, m.shape[1] + gap), float("nan"), dtype=dtype, device=DEV)
        wide[:, :m.shape[1]] = on_gpu(m, dtype)
        return wide[:, :m.shape[1]]
    for form in ("runs", "any"):
        ids = who(rng, T, n, form)
        i = on_gpu(ids, torch.int32)
        Y, Ug = dab.dab_adapters(apart(X), i, a, b, s, base=apart(base))
        Yo, Uo = oa.adapters(X, ids, A, B, scale, base)
        assert np.array_equal(f64(Ug), Uo) and torch.equal(Y, on_gpu(Yo, dtype))
        dX, dA, dB = dab.dab_adapters_gradient(apart(dY), apart(X), Ug, i, a, b, s, base=apart(dbase))
        dXo, dAo, dBo = oa.adapters_gradient(dY, X, Uo, ids, A, B, scale, dbase)
        assert torch.equal(dX, on_gpu(dXo, dtype)) and np.array_equal(f64(dA), dAo) and np.array_equal(f64(dB), dBo)


def test_more_tiles_of_tokens_than_a_grid_has_along_one_dimension():
    T, K, F, n, r = 600001, 16, 8, 2, 65                           # (a rank of two row blocks: U and Y in launches of their own)
    g = torch.Generator(device=DEV).manual_seed(5)
    X, A, B = (torch.randint(-2, 3, s, generator=g, device=DEV).bfloat16() for s in ((T, K), (n, r, K), (n, r, F)))
    ids = torch.randint(-1, n, (T // 37 + 1,), generator=g, device=DEV).repeat_interleave(37)[:T].int()
    base = torch.randint(-9, 10, (T, F), generator=g, device=DEV).bfloat16()
    Y, Ug = dab.dab_adapters(X, ids, A, B, base=base)
    for i in range(n):
        at = torch.nonzero(ids == i).squeeze(1)
        u = X[at].float() @ A[i].float().t()
        assert torch.equal(Ug[at], u) and torch.equal(Y[at], (base[at].float() + u @ B[i].float()).bfloat16())
    none = ids < 0
    assert torch.equal(Y[none], base[none]) and not Ug[none].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [5, 100])
def test_infinities_stay_with_their_tokens(dtype, T):
    rng = np.random.default_rng(6)
    K, F, n, r = 70, 150, 3, 5
    X, A, B, dY, scale, base, dbase = (t.clone() for t in random_values(rng, T, K, F, n, r, dtype))
    ids = rng.integers(0, 2, T).astype(np.int32)
    ids[3], ids[4] = -1, 2
    i = on_gpu(ids, torch.int32)
    clean = dab.dab_adapters(X, i, A, B, scale, base=base)
    grads = dab.dab_adapters_gradient(dY, X, clean[1], i, A, B, scale, base=dbase)
    # adapter 2's matrices and scale, and what token 3 (without an adapter) and token 4 (adapter 2) hold
    A[2], B[2], scale[2] = float("nan"), float("inf"), float("nan")
    X[3], dY[3], X[4, 1] = float("nan"), float("inf"), float("inf")
    Y, Ug = dab.dab_adapters(X, i, A, B, scale, base=base)
    others = torch.tensor([t for t in range(T) if t != 4], device=DEV)
    assert torch.equal(Y[others], clean[0][others]) and torch.equal(Ug[others], clean[1][others]) and bool(Y[4].isnan().all())
    assert torch.equal(Y[3], base[3])
    dX, dA, dB = dab.dab_adapters_gradient(dY, X, Ug, i, A, B, scale, base=dbase)
    assert torch.equal(dX[others], grads[0][others]) and torch.equal(dA[:2], grads[1][:2]) and torch.equal(dB[:2], grads[2][:2])
    assert bool(dA[2].isnan().all()) and bool(dB[2].isnan().all())


@pytest.mark.parametrize("dtype", TYPES)
def test_in_place_and_nothing_behind(dtype):
    rng = np.random.default_rng(7)
    for T in (3, 90):
        K, F, n, r = 45, 83, 2, 6
        X, A, B, dY, scale, base, dbase = random_values(rng, T, K, F, n, r, dtype)
        i = on_gpu(who(rng, T, n, "any"), torch.int32)
        Y, Ug = dab.dab_adapters(X, i, A, B, scale, base=base)
        dX, dA, dB = dab.dab_adapters_gradient(dY, X, Ug, i, A, B, scale, base=dbase)

        def room(shape, t):
            whole = torch.full((int(np.prod(shape)) + 64,), 7.0, dtype=t, device=DEV)
            return whole, whole[:-64].view(shape)
        outs = [room((T, F), dtype), room((T, r), torch.float32), room((T, K), dtype), room((n, r, K), torch.float32), room((n, r, F), torch.float32)]
        outs[0][1].copy_(base), outs[2][1].copy_(dbase)
        dab.dab_adapters(X, i, A, B, scale, base=outs[0][1], out=(outs[0][1], outs[1][1]))
        dab.dab_adapters_gradient(dY, X, outs[1][1], i, A, B, scale, base=outs[2][1], out=tuple(o[1] for o in outs[2:]))
        for o, want in zip(outs, (Y, Ug, dX, dA, dB)):
            assert torch.equal(o[1], want) and bool((o[0][-64:] == 7).all())


def test_gradient_by_differences():
    rng = np.random.default_rng(8)
    T, K, F, n, r = 70, 20, 24, 2, 3
    X, A, B, dY, scale, _, _ = random_values(rng, T, K, F, n, r, torch.float32)
    i = on_gpu(who(rng, T, n, "any"), torch.int32)
    _, Ug = dab.dab_adapters(X, i, A, B, scale)
    got = dab.dab_adapters_gradient(dY, X, Ug, i, A, B, scale)
    for at, grad in ((X, got[0]), (A, got[1]), (B, got[2])):
        d = torch.randn(at.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
        sides = []
        for h in (0.5, -0.5):                                       # bilinear in each: a central difference of any size is exact
            at.add_(d, alpha=h)
            sides.append((dab.dab_adapters(X, i, A, B, scale)[0].double() * dY.double()).sum())
            at.sub_(d, alpha=h)
        want, have = float(sides[0] - sides[1]), float((grad.double() * d.double()).sum())
        size = float((dab.dab_adapters(X.abs() + d.abs().max(), i, A.abs() + d.abs().max(), B.abs() + d.abs().max(), scale)[0].double() * dY.abs().double()).sum())
        assert abs(want - have) <= (K + F + T + 20) * U * 4 * size


def test_offsets_past_32_bits():
    T, ld, K, F, r = 70000, 32768, 40, 24, 4                        # 2.3e9 elements between the first token and the last
    wide = torch.empty((T, ld), dtype=torch.bfloat16, device=DEV)
    X = wide[:, 64:64 + K]
    X.normal_()
    g = torch.Generator(device=DEV).manual_seed(2)
    A, B = (torch.randn((2, r, c), generator=g, device=DEV).bfloat16() for c in (K, F))
    ids = torch.randint(-1, 2, (T // 100,), generator=g, device=DEV).repeat_interleave(100).int()
    dY = torch.randn((T, F), generator=g, device=DEV).bfloat16()
    one, two = dab.dab_adapters(X, ids, A, B), dab.dab_adapters(X.contiguous(), ids, A, B)
    assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
    p, q = dab.dab_adapters_gradient(dY, X, one[1], ids, A, B), dab.dab_adapters_gradient(dY, X.contiguous(), one[1], ids, A, B)
    assert all(torch.equal(a, b) for a, b in zip(p, q))
    tail = f64(one[0][-50:])
    want, _ = oa.adapters(f64(X[-50:]), ids[-50:].cpu().numpy(), f64(A), f64(B), np.ones(2), None)
    assert np.all(np.abs(tail - want) <= 2.0 ** -7 * (np.abs(want) + 1))


# ------------------------------------------------------------------ with 4-bit weights
SERVE = [(1, 128, 16, 1, 1), (1, 500, 100, 3, 16), (2, 64, 33, 2, 4), (7, 911, 409, 3, 8), (16, 256, 64, 20, 16), (31, 640, 130, 4, 33), (48, 130, 272, 5, 64),
         (64, 200, 150, 9, 12), (65, 256, 128, 3, 16), (100, 1030, 48, 2, 5), (200, 96, 300, 70, 7)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,K,F,n,r", SERVE)
def test_served(dtype, T, K, F, n, r):
    rng = np.random.default_rng(T + K + F + n + r + 2)
    X, A, B, _, scale, _, _ = whole_numbers(rng, T, K, F, n, r)
    W = rng.choice([-6.0, -4, -3, -2, -1.5, -1, -0.5, 0, 0.5, 1, 1.5, 2, 3, 4, 6], (F, K))
    W[:, ::32] = 6
    Q, S = dab.dab_w4_pack(on_gpu(W, torch.float32))
    x, a, b, s = on_gpu(X, dtype), on_gpu(A, dtype), on_gpu(B, dtype), on_gpu(scale, torch.float32)
    for form in ("any", "one", "none"):
        ids = who(rng, T, n, form)
        want, _ = oa.adapters(X, ids, A, B, scale, X @ W.T)
        for xs in (x, strided(x, 3, 0), strided(x, 16, 8)):
            Y = dab.dab_w4_adapters(xs, Q, S, F, on_gpu(ids, torch.int32), a, b, s)
            assert Y.dtype == dtype and torch.equal(Y, on_gpu(want, dtype))
    # random values: products of 4-bit weights are exact in pieces, so the sums round once a term
    X, A, B, _, scale, _, _ = random_values(rng, T, K, F, n, r, dtype)
    Q, S = dab.dab_w4_pack(on_gpu(rng.standard_normal((F, K)), torch.float32))
    W = f64(dab.dab_w4_unpack(Q, S, F, K))
    ids = who(rng, T, n, "any")
    Y = dab.dab_w4_adapters(X, Q, S, F, on_gpu(ids, torch.int32), A, B, scale)
    want, _ = oa.adapters(f64(X), ids, f64(A), f64(B), f64(scale), f64(X) @ W.T)
    size, _ = oa.adapters(np.abs(f64(X)), ids, np.abs(f64(A)), np.abs(f64(B)), f64(scale), np.abs(f64(X)) @ np.abs(W).T)
    off = (3 * K + r + 8) * U * size
    assert np.all(np.abs(f64(Y) - want) <= off + HALF[dtype] * (np.abs(want) + off))


def test_served_tokens_keep_to_themselves():
    rng = np.random.default_rng(9)
    T, K, F, n, r = 6, 256, 64, 3, 4
    X, A, B, _, scale, _, _ = random_values(rng, T, K, F, n, r, torch.bfloat16)
    Q, S = dab.dab_w4_pack(on_gpu(rng.standard_normal((F, K)), torch.float32))
    ids = on_gpu(np.array([0, 1, 2, -1, 1, 0], dtype=np.int32), torch.int32)
    clean = dab.dab_w4_adapters(X, Q, S, F, ids, A, B, scale)
    A[2], B[2], X[2, 0] = float("nan"), float("inf"), float("inf")
    Y = dab.dab_w4_adapters(X, Q, S, F, ids, A, B, scale)
    for t in range(T):
        assert torch.equal(Y[t], clean[t]) if t != 2 else bool(Y[t].isnan().all())
    # without an adapter it is the product alone, its sums in another order: a step of bf16 apart at most
    alone = dab.dab_w4_matvec(X[3:4], Q, S, F)[0]
    assert bool(((Y[3].float() - alone.float()).abs() <= 2.0 ** -7 * alone.float().abs() + (3 * K + 8) * U * f64(X[3:4].abs()).sum() * 6).all())


# ------------------------------------------------------------------ graphs, streams, refusals
def test_captured_and_on_another_stream():
    rng = np.random.default_rng(10)
    T, K, F, n, r = 150, 130, 200, 3, 8
    X, A, B, dY, scale, base, dbase = random_values(rng, T, K, F, n, r, torch.bfloat16)
    Q, S = dab.dab_w4_pack(on_gpu(rng.standard_normal((F, K)), torch.float32))
    i = on_gpu(who(rng, T, n, "any"), torch.int32)
    outs = [torch.empty_like(base), torch.empty((T, r), device=DEV), torch.empty_like(dbase), torch.empty((n, r, K), device=DEV), torch.empty((n, r, F), device=DEV),
            torch.empty_like(base[:9])]
    ws = torch.empty(dab.lib().dab_adapters_gradient_workspace_bytes(T, K, F, n, r), dtype=torch.uint8, device=DEV)
    ws2 = torch.empty(dab.lib().dab_w4_adapters_workspace_bytes(9, K, F, r, dab.DAB_BF16, K), dtype=torch.uint8, device=DEV)

    def work():
        dab.dab_adapters(X, i, A, B, scale, base=base, out=tuple(outs[:2]))
        dab.dab_adapters_gradient(dY, X, outs[1], i, A, B, scale, base=dbase, out=tuple(outs[2:5]), ws=ws)
        dab.dab_w4_adapters(X[:9], Q, S, F, i[:9], A, B, scale, out=outs[5], ws=ws2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for k in range(4):
        X.normal_(), dY.normal_()
        i.copy_(on_gpu(who(rng, T, n, ("any", "one", "none", "runs")[k]), torch.int32))
        graph.replay()
        got = [t.clone() for t in outs]
        Y, Ug = dab.dab_adapters(X, i, A, B, scale, base=base)
        want = [Y, Ug, *dab.dab_adapters_gradient(dY, X, Ug, i, A, B, scale, base=dbase), dab.dab_w4_adapters(X[:9], Q, S, F, i[:9], A, B, scale)]
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        torch.cuda.synchronize()


def test_refusals():
    rng = np.random.default_rng(11)
    T, K, F, n, r = 5, 40, 24, 2, 3
    X, A, B, dY, scale, base, dbase = random_values(rng, T, K, F, n, r, torch.bfloat16)
    ids = on_gpu(who(rng, T, n, "any"), torch.int32)
    good = dict(X=X, ids=ids, A=A, B=B, scale=scale, base=base)
    wide = torch.zeros((n, 257, K), dtype=torch.bfloat16, device=DEV)
    for bad, error in ((dict(X=X.cpu()), TypeError), (dict(ids=ids.long()), TypeError), (dict(ids=ids[:4]), ValueError), (dict(A=A.float()), TypeError),
                       (dict(B=B[:1]), ValueError), (dict(A=A[0]), ValueError), (dict(scale=scale[:1]), ValueError), (dict(base=base.half()), TypeError),
                       (dict(base=base[:, :5]), ValueError), (dict(A=wide, B=torch.zeros((n, 257, F), dtype=torch.bfloat16, device=DEV)), dab.DabError),
                       (dict(X=X[:0], ids=ids[:0], base=None), dab.DabError), (dict(X=X[:, 1:], A=A[:, :, 1:].contiguous()), dab.DabError)):
        with pytest.raises(error):
            dab.dab_adapters(**{**good, **bad})
    _, Ug = dab.dab_adapters(**good)
    grads = dict(dY=dY, X=X, U=Ug, ids=ids, A=A, B=B, scale=scale, base=dbase)
    with pytest.raises(dab.DabError):
        dab.dab_adapters_gradient(**grads, out=(X, None, None))     # X is read again behind dX
    for bad, error in ((dict(dY=None), TypeError), (dict(dY=dY.half()), TypeError), (dict(U=Ug[:, :2]), ValueError), (dict(base=base), ValueError),
                       (dict(want_dX=False), ValueError)):
        with pytest.raises(error):
            dab.dab_adapters_gradient(**{**grads, **bad})
    Q, S = dab.dab_w4_pack(on_gpu(rng.standard_normal((F, K)), torch.float32))
    with pytest.raises(ValueError):
        dab.dab_w4_adapters(X, Q, S, F + 16, ids, A, B, scale)
    with pytest.raises(ValueError):
        dab.dab_w4_adapters(X, Q[:1], S, F, ids, A, B, scale)
