"""The tokens' weights in the head's gradient: one weight for all tokens (a mean's 1/N) scales dH and dW in fp32, whatever the type of H and W."""
import pytest
import torch

from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U16 = 2.0 ** -8                            # a number rounded to bf16, relative (8 bits: half of 2^-7)
# bf16 heads of more than 128 tokens on tiles: one piece of the vocabulary and several, shares of the sums, rows that are no whole pieces of 16 bytes
TILES = [(300, 256, 5000), (129, 2000, 9001), (2000, 1024, 8000), (4100, 64, 70001), (5000, 130, 5000), (300, 255, 5000), (8200, 66, 6000), (2048, 512, 32768)]
OTHERS = [(100, 256, 5000), (200, 64, 250), (1, 64, 5000)]      # up to 128 tokens, small heads: P has 16 or 24 bits


def case(T, D, V):
    g = torch.Generator(device=DEV).manual_seed(T + D + V)
    H = torch.randn((T, D), generator=g, device=DEV).bfloat16()
    W = (torch.randn((V, D), generator=g, device=DEV) + 8 * torch.randn((1, D), generator=g, device=DEV)) * (2 / D ** 0.5)
    t = torch.randint(0, V, (T,), generator=g, device=DEV)
    t[1::9] = -100
    return H, W.bfloat16(), t, g


@pytest.mark.parametrize("weight", [1.00390625, 1.0 / 1843, -0.3, 1e-30])
@pytest.mark.parametrize("T,D,V", TILES)
def test_one_weight_for_all_scales_the_gradient(T, D, V, weight):
    """Both results are sums of the same terms but for a factor, in fp32, rounded once.  (1 + 2^-8 lies in the middle of two bf16 numbers: with the
    targets' terms alone rounded to either, what words have in common would stay in dH.)"""
    H, W, t, _ = case(T, D, V)
    _, lse = dab.dab_head_loss(H, W, t)
    ones = dab.dab_head_loss_gradient(H, W, t, lse)
    g = torch.full((T,), weight, device=DEV)
    g[t == -100] = float("nan")                                    # (weights of ignored tokens may be anything)
    weight = float(torch.tensor(weight, dtype=torch.float32))
    live = (t != -100)[:, None]
    h, w = torch.where(live, H.float(), 0.0).abs(), W.float().abs()
    P = torch.softmax(torch.where(live, H.float(), 0.0) @ W.float().t(), 1)
    P[torch.arange(T, device=DEV), t.clamp(min=0)] -= 1
    P = torch.where(live, P.abs(), 0.0)
    # (either result rounds every addition once, by 2^-24 of what the terms amount to; entries of P below 2^-126 have steps of 2^-133)
    sizes = (P @ w, w.sum(dim=0)[None], V), (P.t().contiguous() @ h, h.sum(dim=0)[None], T)
    for got, one, (size, others, terms) in zip(dab.dab_head_loss_gradient(H, W, t, lse, g), ones, sizes):
        want = one.double() * weight
        limit = 2.02 * U16 * want.abs() + 2 * (terms + 4) * 2.0 ** -24 * abs(weight) * size.double() + 2.0 ** -133 * (1 + others.double())
        assert bool(((got.double() - want).abs() <= limit).all())


@pytest.mark.parametrize("T,D,V", [(300, 256, 5000), (2500, 130, 5000)])
def test_tokens_of_no_weight_beside_others_of_one(T, D, V):
    """The first 1100 tokens, or half of the first ones, and every third after them have weight 0."""
    H, W, t, _ = case(T, D, V)
    mask = torch.ones((T,), device=DEV)
    mask[:min(1100, T // 2)] = 0
    mask[::3] = 0
    _, lse = dab.dab_head_loss(H, W, t)
    for got, one in zip(dab.dab_head_loss_gradient(H, W, t, lse, mask * 1.00390625), dab.dab_head_loss_gradient(H, W, t, lse, mask)):
        # (two roundings of up to 2^-8, 2^-8 / sqrt(3) in the mean at most: 0.0032)
        assert float((got.double() - one.double() * 1.00390625).norm()) <= U16 * float(one.double().norm())


@pytest.mark.parametrize("T,D,V", OTHERS)
def test_one_weight_for_all_of_other_heads(T, D, V):
    H, W, t, _ = case(T, D, V)
    _, lse = dab.dab_head_loss(H, W, t)
    ones = dab.dab_head_loss_gradient(H, W, t, lse)
    for got, one in zip(dab.dab_head_loss_gradient(H, W, t, lse, torch.full((T,), 1.00390625, device=DEV)), ones):
        want = one.double() * 1.00390625
        assert float((got.double() - want).norm()) <= U16 * float(want.norm())


SPECIAL = {"zero": [0.0], "some zero": [0.0, 0.7], "infinite": [float("inf"), 0.5], "undefined": [float("nan"), 0.5], "far apart": [1e-20, 1e20], "both signs": [-0.9, 0.1]}


@pytest.mark.parametrize("kind", SPECIAL)
@pytest.mark.parametrize("T,D,V", [(300, 256, 5000), (4100, 64, 70001)])
def test_weights_of_any_kind(T, D, V, kind):
    """Against float64, token by token: a token's row of dH has its own weight, and NaN or infinite where that is."""
    H, W, t, gen = case(T, D, V)
    W = (W.float() - W.float().mean(dim=0)).bfloat16()             # (nothing in common: sums do not cancel)
    g = torch.tensor(SPECIAL[kind], device=DEV).repeat(T)[:T].contiguous()
    _, lse = dab.dab_head_loss(H, W, t)
    dH, dW = dab.dab_head_loss_gradient(H, W, t, lse, g)
    live = t != -100
    fine = live & torch.isfinite(g)
    h, w = H.double(), W.double()
    P = torch.softmax(h @ w.t().contiguous(), 1)
    P[torch.arange(T, device=DEV), t.clamp(min=0)] -= 1
    want = (P @ w) * g.double()[:, None]
    rows = (dH.double() - want)[fine].norm(dim=1), want[fine].norm(dim=1)
    assert bool((rows[0] <= 1e-2 * rows[1]).all())                 # (a row's own roundings: 2^-8 of P's largest entry, 2^-8 of the row)
    assert not bool(dH[~live].any()) and not bool(torch.isfinite(dH[live & ~fine]).any())
    P = P * g.double()[:, None]
    P[~live] = 0
    if bool(fine[live].all()):
        ref = P.t().contiguous() @ h
        assert float((dW.double() - ref).norm()) <= 6e-3 * float(ref.norm()) if kind != "zero" else not bool(dW.any())
