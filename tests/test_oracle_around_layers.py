"""The definitions of norms, 8-bit states, steps and adapters, against differences, identities and each other (no GPU)."""
import numpy as np
import pytest

from oracle import around_layers as oa


@pytest.mark.parametrize("with_dh", [False, True])
def test_norm_gradient_is_that_of_the_norm(with_dh):
    rng = np.random.default_rng(1)
    h, dy, gain = rng.standard_normal((3, 7)), rng.standard_normal((3, 7)), rng.standard_normal(7)
    dh = rng.standard_normal((3, 7)) if with_dh else None
    eps, d = 0.1, 1e-6

    def value(h, gain):
        return float((oa.rms_norm(h, gain, eps)[0] * dy).sum() + (0 if dh is None else (h * dh).sum()))
    dx, dgain = oa.rms_norm_gradient(dy, h, gain, oa.rms_norm(h, gain, eps)[1], dh)
    for r in range(3):
        for c in range(7):
            e = np.zeros((3, 7))
            e[r, c] = d
            assert abs((value(h + e, gain) - value(h - e, gain)) / (2 * d) - dx[r, c]) < 1e-7
    for c in range(7):
        e = np.zeros(7)
        e[c] = d
        assert abs((value(h, gain + e) - value(h, gain - e)) / (2 * d) - dgain[c]) < 1e-7


def test_adapters_gradient_is_that_of_the_adapters():
    rng = np.random.default_rng(2)
    T, K, F, n, r = 5, 4, 6, 2, 3
    X, A, B = rng.standard_normal((T, K)), rng.standard_normal((n, r, K)), rng.standard_normal((n, r, F))
    dY, scale, ids = rng.standard_normal((T, F)), np.array([0.5, 2.0]), np.array([1, -1, 0, 1, 7])

    def value(X, A, B):
        return float((oa.adapters(X, ids, A, B, scale, None)[0] * dY).sum())
    U = oa.adapters(X, ids, A, B, scale, None)[1]
    got = oa.adapters_gradient(dY, X, U, ids, A, B, scale, None)
    for k, at in enumerate((X, A, B)):
        for i in np.ndindex(at.shape):
            sides = []
            for d in (1e-6, -1e-6):
                moved = [X.copy(), A.copy(), B.copy()]
                moved[k][i] += d
                sides.append(value(*moved))
            assert abs((sides[0] - sides[1]) / 2e-6 - got[k][i]) < 1e-7
    assert not got[0][1].any() and not got[0][4].any()


@pytest.mark.parametrize("is_signed", [True, False])
def test_values_of_a_state_keep_their_codes(is_signed):
    levels = oa.state_values(3 if is_signed else 4)
    assert np.all(np.diff(levels) > 0) and levels[0] == 0 and levels[-1] < 2
    # a group whose largest value is below 2 and at least 1 has scale 2^0; the smallest chance rounds down, so codes keep themselves
    for at in range(0, len(levels), 31):
        x = np.concatenate([[1.5], levels[at:at + 31]]).astype(np.float32)
        for c in (0, 65535):
            codes, scales = oa.state_save(x, np.full(32, c), is_signed)
            assert scales[0] == 127 and np.array_equal(oa.state_restore(codes, scales, is_signed)[:len(x)], x)


@pytest.mark.parametrize("is_signed", [True, False])
def test_rounding_by_chance_keeps_the_mean(is_signed):
    rng = np.random.default_rng(3)
    x = (np.abs(rng.standard_normal(32)) * np.exp(2 * rng.standard_normal(32))).astype(np.float32)
    x[0] = 1.99 * 2.0 ** np.ceil(np.log2(np.max(x)))               # (above the last code of its binade)
    chances = np.arange(0, 65536, 257)                              # 256 of them, evenly spread
    total = np.zeros(32)
    for c in chances:
        total += oa.state_restore(*oa.state_save(x, np.full(32, c), is_signed), is_signed)
    levels = oa.state_values(3 if is_signed else 4)
    f = 2.0 ** (np.floor(np.log2(np.max(x))) + 1)
    for i in range(32):
        y = x[i] / f
        at = min(np.searchsorted(levels, y, side="right") - 1, len(levels) - 2)
        step = (levels[at + 1] - levels[at]) * f
        # off by one of 256 chances, and by what a code of at least 1 adds to roots below half of the smallest
        assert abs(total[i] / len(chances) - x[i]) <= step / 250 + (0 if is_signed or y >= levels[1] else levels[1] * f)


def test_chances_are_spread_evenly_and_differ():
    c = np.array([oa.chance(5, 1, i) for i in range(4096)])
    for part in (c & 0xFFFF, c >> 16):
        # the mean of 4096 uniform numbers: 5 standard deviations of 1 / sqrt(12 * 4096)
        assert abs(np.mean(part) / 65536 - 0.5) < 5 / np.sqrt(12 * 4096)
        assert abs(np.corrcoef(part[:-1], part[1:])[0, 1]) < 5 / np.sqrt(4096)
    assert abs(np.corrcoef(c & 0xFFFF, c >> 16)[0, 1]) < 5 / np.sqrt(4096)
    other = np.array([oa.chance(5, 2, i) for i in range(4096)])
    assert abs(np.corrcoef(c, other)[0, 1]) < 5 / np.sqrt(4096) and oa.chance(5, 1, 1 << 32) != oa.chance(5, 1, 0)


def test_a_step_is_that_of_its_formula():
    rng = np.random.default_rng(4)
    p, g, m = (rng.standard_normal(50).astype(np.float32) for _ in range(3))
    v = (rng.standard_normal(50) ** 2).astype(np.float32)
    got = oa.adamw(p, g, m, v, 1e-2, 3, 0.9, 0.99, 1e-8, 0.1, 0.5)
    g64, m64, v64 = 0.5 * g.astype(float), m.astype(float), v.astype(float)
    m64, v64 = 0.9 * m64 + 0.1 * g64, 0.99 * v64 + 0.01 * g64 ** 2
    want = p * (1 - 1e-2 * 0.1) - 1e-2 * (m64 / (1 - 0.9 ** 3)) / (np.sqrt(v64 / (1 - 0.99 ** 3)) + 1e-8)
    np.testing.assert_allclose(got[0], want, rtol=0, atol=8 * 2.0 ** -24 * (np.max(np.abs(p)) + 0.1))
