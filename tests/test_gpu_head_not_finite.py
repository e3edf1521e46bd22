"""Words and tokens of the head that are no numbers: a loss that any of its logits leaves undefined is NaN, and so is lse, whichever kernels a
head's sizes choose and however the words fall into their blocks (of 32, 64 or 128)."""
import pytest
import torch

from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
NAN = float("nan")
# (tokens, width, words): one word behind a whole number of blocks, of every kind of kernel
SMALL, FEW, MANY = (5, 16, 129), (33, 64, 4225), (2100, 1024, 4225)
CASES = [(torch.bfloat16, SMALL), (torch.bfloat16, FEW), (torch.bfloat16, MANY), (torch.bfloat16, (1, 512, 131073)),
         (torch.float32, SMALL), (torch.float32, FEW), (torch.float32, MANY), (torch.float32, (1, 64, 5121))]


def case(dtype, sizes):
    T, D, V = sizes
    g = torch.Generator(device=DEV).manual_seed(T + V)
    H = torch.randn((T, D), generator=g, device=DEV).to(dtype)
    W = (torch.randn((V, D), generator=g, device=DEV) / D ** 0.5).to(dtype)
    t = torch.randint(0, V // 2, (T,), generator=g, device=DEV)
    t[1::5] = -100
    return H, W, t


# words of W that diverged: the last one, alone in its block; one block; all of a token's blocks but the first ones; one in the middle
WORDS = {"last": slice(-1, None), "block": slice(-129, -1), "most": slice(65, None), "one": slice(70, 71)}


@pytest.mark.parametrize("words", WORDS)
@pytest.mark.parametrize("dtype,sizes", CASES)
def test_diverged_words_show_in_the_loss(dtype, sizes, words):
    H, W, t = case(dtype, sizes)
    W[WORDS[words]] = NAN
    loss, lse = dab.dab_head_loss(H, W, t)
    live = t != -100
    assert bool(torch.isnan(loss[live]).all()) and bool(torch.isnan(lse[live]).all())
    assert not bool(loss[~live].any()) and not bool(lse[~live].any())
    dH, _ = dab.dab_head_loss_gradient(H, W, t, lse)
    assert bool(torch.isnan(dH[live]).all())


@pytest.mark.parametrize("dtype,sizes", CASES)
def test_a_diverged_token_shows_in_its_own_loss_only(dtype, sizes):
    H, W, t = case(dtype, sizes)
    loss, lse = dab.dab_head_loss(H, W, t)
    H[0] = NAN
    if sizes[0] > 4:
        H[4, 3] = NAN
    bad = torch.isnan(H).any(dim=1)
    got, got_lse = dab.dab_head_loss(H, W, t)
    assert bool(torch.isnan(got[bad]).all()) and bool(torch.isnan(got_lse[bad]).all())
    assert torch.equal(got[~bad], loss[~bad]) and torch.equal(got_lse[~bad], lse[~bad])


def no_weight(dtype, sizes):
    """(loss, lse) of words half of which have logits of minus infinity, float64's, and what rounding allows."""
    T, D, V = sizes
    H, W, t = case(dtype, sizes)
    H, W = H.abs() + 0.5, W.abs()                                 # (a product with minus infinity is minus infinity)
    kept = V // 2
    L = H.double() @ W[:kept].double().t()
    ref = torch.logsumexp(L, 1)
    W[kept:] = float("-inf")
    live = t != -100
    want = ref - L.gather(1, t.clamp(min=0)[:, None])[:, 0]
    loss, lse = dab.dab_head_loss(H, W, t)
    return loss[live].double(), lse[live].double(), want[live], ref[live], 2e-5 * max(1.0, float(L.abs().max()))


@pytest.mark.parametrize("dtype,sizes", [c for c in CASES if c != (torch.float32, MANY)])
def test_words_of_no_weight_add_nothing(dtype, sizes):
    """Logits of minus infinity, whole blocks of them: their words have probability 0, and the loss is that of the others."""
    loss, lse, want, ref, tol = no_weight(dtype, sizes)
    assert bool(((lse - ref).abs() <= tol).all()) and bool(((loss - want).abs() <= tol).all())


def test_infinities_among_fp32_words_never_give_a_wrong_number():
    """Products of pieces have no infinite logits: an infinity's products with the pieces of a number have both signs, or are undefined."""
    loss, lse, want, ref, tol = no_weight(torch.float32, MANY)
    assert bool((((lse - ref).abs() <= tol) | torch.isnan(lse)).all()) and bool((((loss - want).abs() <= tol) | torch.isnan(loss)).all())


# and a vocabulary in several pieces, with and without shares of dH's sums
IGNORED = CASES + [(torch.bfloat16, (4100, 64, 70001)), (torch.bfloat16, (70000, 40, 4099)), (torch.bfloat16, (129, 2000, 9001)), (torch.float32, (4100, 64, 70001))]


@pytest.mark.parametrize("value", [NAN, float("inf")])
@pytest.mark.parametrize("dtype,sizes", IGNORED)
def test_tokens_without_a_loss_have_no_gradient_whatever_the_words_hold(dtype, sizes, value):
    T, D, V = sizes
    H, W, t = case(dtype, sizes)
    t[2::7] = V
    t[3::11] = -1
    t[-1] = -100
    W[V // 3] = value
    _, lse = dab.dab_head_loss(H, W, t)
    dH, _ = dab.dab_head_loss_gradient(H, W, t, lse)
    dead = (t < 0) | (t >= V)
    assert not bool(dH[dead].any()) and not bool(torch.isfinite(dH[~dead]).any())
