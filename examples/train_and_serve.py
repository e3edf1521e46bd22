"""A binarized layer under a large real head: trained, then served with the head in 4 bits.

    python examples/train_and_serve.py [steps]

The layer's weights are binarized every step (mean-centred, clamped, split: Algorithm 2), its inputs are real.  What its backward pass
needs of them is kept in 8 bits.  The head's loss is taken without the logits, and so are its gradients:

    forward    W~ from W;  Y = X W~^T;  X kept as bytes;  loss of H V^T, H = Y in bf16
    backward   dH, dV of the loss;  dW~ = dH^T X from the bytes;  the gradient of W by Theorem 4's factor
    serving    V laid out in 4 bits once;  each token one product with W~ and one with the 4-bit head

Inputs and targets are synthetic: a teacher of the same shape names the word for each input.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1804_02941_amd import binding as dab  # noqa: E402

DEV = "cuda:0"
INPUTS, WIDTH, WORDS, TOKENS = 512, 256, 5000, 1024


def batch(teacher, g, tokens=TOKENS):
    """Inputs fp32 [tokens, INPUTS] and their words; one token in ten has none (-100)."""
    X = torch.randn((tokens, INPUTS), generator=g, device=DEV)
    words = (torch.tanh(X @ teacher[0].t()) @ teacher[1].t()).argmax(dim=1)
    words[torch.rand(tokens, generator=g, device=DEV) < 0.1] = -100
    return X, words


def binarize(W):
    """The layer's weights as the binarized layer takes them."""
    centred = dab.dab_mean_center_clamp(W.view(WIDTH, INPUTS, 1, 1)).view(WIDTH, INPUTS)
    est = dab.dab_estimate_alpha_beta(centred)
    E, _ = dab.dab_pack_weights(centred.view(WIDTH, INPUTS, 1, 1), est["thr_val"], est["thr_idx"], est["alpha_is_upper"])
    return centred, est, E


def step(W, V, X, words, rate):
    """One step of gradient descent on W (fp32) and V (an fp32 master of the bf16 head); returns the mean loss."""
    centred, est, E = binarize(W)
    H = dab.dab_wbin_fc(X, E, est["alpha"], est["beta"]).bfloat16()
    saved = dab.dab_ckpt8_save(X)
    head = V.bfloat16()
    loss, lse = dab.dab_head_loss(H, head, words)
    live = words != -100
    weight = live.float() / live.sum()
    dH, dV = dab.dab_head_loss_gradient(H, head, words, lse, weight)
    dWt = dab.dab_ckpt8_weight_gradient(dH, *saved, INPUTS)
    dW = dab.dab_weight_gradient(centred, est["thr_val"], est["thr_idx"], est["alpha_is_upper"], upstream=dWt)
    W -= rate * dW
    V -= rate * dV.float()
    return (loss * weight).sum()


def serve(W, V4, X):
    """The words that the trained network answers with, one token at a time; V4: the head as dab_w4_pack() lays it out."""
    _, est, E = binarize(W)
    answers = []
    for x in X.split(1):
        H = dab.dab_wbin_fc(x, E, est["alpha"], est["beta"])
        answers.append(dab.dab_w4_matvec(H, *V4, WORDS).argmax(dim=1))
    return torch.cat(answers)


def main(steps=200, rate=30.0, seed=1):
    """Trains and serves; returns (first and last mean loss, share of served words that the bf16 head would have answered)."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    teacher = (torch.randn((WIDTH, INPUTS), generator=g, device=DEV) / INPUTS ** 0.5, torch.randn((WORDS, WIDTH), generator=g, device=DEV))
    W = torch.randn((WIDTH, INPUTS), generator=g, device=DEV) / INPUTS ** 0.5
    V = 0.02 * torch.randn((WORDS, WIDTH), generator=g, device=DEV)
    losses = []
    for i in range(steps):
        loss = step(W, V, *batch(teacher, g), rate)
        if i % 20 == 0 or i == steps - 1:
            losses.append(float(loss))
            print(f"step {i:4d}  loss {losses[-1]:.3f}", flush=True)
    X, _ = batch(teacher, g, 64)
    served = serve(W, dab.dab_w4_pack(V), X)
    _, est, E = binarize(W)
    real = (dab.dab_wbin_fc(X, E, est["alpha"], est["beta"]) @ V.t()).argmax(dim=1)
    same = float((served == real).float().mean())
    print(f"served with a 4-bit head: {100 * same:.0f} % of the answers are those of the fp32 head")
    return losses[0], losses[-1], same


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
