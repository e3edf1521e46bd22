"""A frozen 4-bit layer that learns several tasks by adapters, then serves requests of all of them together.

    python examples/adapt_and_serve.py [steps]

The layer's weights are laid out in 4 bits once and stay as they are.  What is learned is small: a pair of matrices of low rank for every task, and the gain
of the norm in front of the layer, with AdamW's states in 8 bits:

    forward    y = norm(x) * gain;  z = W4 y + scale_i B_i (A_i y) for each token's task i;  the loss of z V^T
    backward   dz of the loss;  dA_i, dB_i and dy;  the gain's gradient;  one step over all tensors
    serving    tokens of any tasks in one call: the 4-bit product and every token's adapter

Inputs and targets are synthetic: a teacher whose layer differs from the frozen one by a change of low rank for each task.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_1804_02941_amd import binding as dab  # noqa: E402

DEV = "cuda:0"
INPUTS, WIDTH, WORDS, TASKS, RANK, TOKENS = 256, 192, 1000, 3, 8, 512


class Model:
    def __init__(self, seed=1):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def normal(*shape, by=1.0):
            return by * torch.randn(shape, generator=g, device=DEV)
        W = normal(WIDTH, INPUTS, by=INPUTS ** -0.5)
        self.Q, self.S = dab.dab_w4_pack(W)
        self.W4 = dab.dab_w4_unpack(self.Q, self.S, WIDTH, INPUTS)      # for the gradient of the layer's input
        self.V = normal(WORDS, WIDTH, by=0.3)
        self.V4 = dab.dab_w4_pack(self.V)
        self.teacher = W + torch.einsum("trf,trk->tfk", normal(TASKS, RANK, WIDTH, by=0.5), normal(TASKS, RANK, INPUTS, by=INPUTS ** -0.5))
        self.gain = torch.ones(INPUTS, device=DEV)
        self.A, self.B = normal(TASKS, RANK, INPUTS, by=INPUTS ** -0.5), torch.zeros((TASKS, RANK, WIDTH), device=DEV)
        self.scale = torch.ones(TASKS, device=DEV)
        self.grads = {k: torch.zeros_like(getattr(self, k)) for k in ("A", "B", "gain")}
        states = {k: dab.adamw_states(getattr(self, k), bits=8) for k in self.grads}
        self.jobs = dab.adamw_jobs([{"P": getattr(self, k), "G": self.grads[k], "M": states[k][0], "V": states[k][1],
                                     "weight_decay": 0.0 if k == "gain" else 0.01} for k in self.grads])
        self.g = g

    def batch(self, tokens=TOKENS):
        """Inputs, the task of each, and the word that the teacher names."""
        X = torch.randn((tokens, INPUTS), generator=self.g, device=DEV)
        tasks = torch.randint(0, TASKS, (tokens,), generator=self.g, device=DEV).int()
        y = X / X.square().mean(dim=1, keepdim=True).sqrt()
        z = torch.stack([y @ w.t() for w in self.teacher])[tasks.long(), torch.arange(tokens, device=DEV)]
        return X, tasks, (z @ self.V.t()).argmax(dim=1)

    def gradients(self, X, tasks, words):
        """The mean loss, and the gradients in self.grads."""
        y, h, rstd, _ = dab.dab_rms_norm(X, self.gain)
        z, U = dab.dab_adapters(y, tasks, self.A, self.B, self.scale, base=dab.dab_w4_matvec(y, self.Q, self.S, WIDTH))
        loss, lse = dab.dab_head_loss(z, self.V, words)
        weight = torch.full((X.shape[0],), 1.0 / X.shape[0], device=DEV)
        dz, _ = dab.dab_head_loss_gradient(z, self.V, words, lse, weight)
        dy, _, _ = dab.dab_adapters_gradient(dz, y, U, tasks, self.A, self.B, self.scale, base=dz @ self.W4, out=(None, self.grads["A"], self.grads["B"]))
        dab.dab_rms_norm_gradient(dy, h, self.gain, rstd, out=(None, self.grads["gain"]))
        return loss.mean()

    def step(self, number, rate):
        loss = self.gradients(*self.batch())
        dab.dab_adamw(self.jobs, rate, number, seed=1)
        return loss

    def serve(self, X, tasks):
        """The words that the model answers with, requests of all tasks together."""
        y, _, _, _ = dab.dab_rms_norm(X, self.gain)
        z = dab.dab_w4_adapters(y, self.Q, self.S, WIDTH, tasks, self.A, self.B, self.scale)
        return dab.dab_w4_matvec(z, *self.V4, WORDS).argmax(dim=1)


def main(steps=200, rate=0.02, seed=1):
    """Trains and serves; returns the share of the served words that are the teacher's."""
    model = Model(seed)
    for i in range(1, steps + 1):
        loss = model.step(i, rate)
        if i % 20 == 1 or i == steps:
            print(f"step {i:4d}  loss {float(loss):.3f}", flush=True)
    X, tasks, words = model.batch(48)
    served = torch.cat([model.serve(x, t) for x, t in zip(X.split(16), tasks.split(16))])
    same = float((served == words).float().mean())
    print(f"served with 4-bit weights and adapters: {100 * same:.0f} % of the answers are the teacher's")
    return same


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 200)
