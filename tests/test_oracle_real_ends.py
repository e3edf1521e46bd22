"""The float64 definitions of saved inputs, 4-bit weights and the loss, against hand examples, a library and differences."""
import numpy as np
import pytest
import torch

from oracle import real_ends as oe


def test_saved_values_by_hand():
    x = np.zeros((1, 40))
    x[0, :4] = [1.0, -2.0, 127.4 / 64, 0.0]                       # largest 2: exponent 1 - 6 = -5, one is 32 steps
    x[0, 32:36] = [1.0, 127.75 / 128, 0.5, 1.5 / 64]              # largest 1: 64 steps
    Q, S = oe.save8(x)
    assert S.tolist() == [[127 - 5, 127 - 6]]
    assert Q[0, :4].tolist() == [32, -64, 64, 0] and Q[0, 32:36].tolist() == [64, 64, 32, 2]
    assert not Q[0, 36:].any()
    y = np.zeros((1, 2))
    y[0] = [255 / 128, 1.0]                                       # 127.5 steps of 2^-6 would round past the last byte
    Q, S = oe.save8(y)
    assert S[0, 0] == 127 - 5 and Q[0, :2].tolist() == [64, 32]


def test_saved_values_are_within_half_a_step_and_bf16_numbers():
    rng = np.random.default_rng(5)
    x = (rng.standard_normal((50, 77)) * np.exp(rng.normal(size=(50, 1)) * 8)).astype(np.float32)
    x[3] = 0
    back = oe.restore8(*oe.save8(x), 77)
    step = np.repeat(np.ldexp(1.0, oe.save8(x)[1].astype(int) - 127), 32, axis=1)[:, :77]
    assert np.all(np.abs(back - x) <= 0.5 * step)
    t = torch.from_numpy(back)
    assert torch.equal(t.bfloat16().double(), t)


def test_4_bit_codes_by_hand():
    w = np.array([[0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.9, -0.0, -7.0]])
    codes, scale = oe.pack4(w)                                    # largest 7: exponent 2 - 2 = 0, ties to the even code
    assert scale[0, 0] == 127
    assert codes[0, :11].tolist() == [0, 1, 2, 2, 4, 4, 6, 6, 7, 8, 15]
    codes, scale = oe.pack4(np.array([[7.25, 1.0]]))              # further from 6 than from 8, which is 4 steps of two
    assert scale[0, 0] == 128 and codes[0, :2].tolist() == [6, 1]


def test_loss_and_gradient_against_the_library_and_differences():
    rng = np.random.default_rng(7)
    T, D, V = 9, 6, 13
    H, W, g = rng.standard_normal((T, D)), rng.standard_normal((V, D)), rng.random(T)
    t = rng.integers(0, V, T)
    t[4] = -100
    loss, lse, P, dH, dW = oe.head(H, W, t, g, -100)
    h, w = (torch.from_numpy(a).requires_grad_() for a in (H, W))
    ref = torch.nn.functional.cross_entropy(h @ w.t(), torch.from_numpy(t), reduction="none", ignore_index=-100)
    (ref * torch.from_numpy(g)).sum().backward()
    np.testing.assert_allclose(loss, ref.detach().numpy(), rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(dH, h.grad.numpy(), rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(dW, w.grad.numpy(), rtol=1e-10, atol=1e-12)
    d = rng.standard_normal((V, D))
    at = [float(g @ oe.head(H, W + s * 1e-5 * d, t, g, -100)[0]) for s in (1, -1)]
    assert (at[0] - at[1]) / 2e-5 == pytest.approx(float(np.sum(dW * d)), rel=1e-7)


def test_layout_of_4_bit_weights_by_hand():
    codes, scale = np.zeros((18, 160), dtype=np.uint8), np.full((18, 5), 17, dtype=np.uint8)
    codes[17, 129], scale[17, 4] = 11, 99                         # row 17, weight 129: tile 1, block 1, group 0, upper half of byte 0
    Q, S = oe.tiles4(codes, scale)
    assert Q.shape == (2, 2, 64, 16) and S.shape == (2, 1, 64, 4)
    assert Q[1, 1, 1, 0] == 11 << 4 and Q.sum() == 11 << 4
    assert S[1, 0, 1, 1] == 99
