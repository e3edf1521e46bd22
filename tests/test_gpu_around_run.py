"""Norms, adapters, the head, 8-bit inputs and steps together, as a fine-tuning step and a server use them, against float64.

A block: h = x + r; y = norm(h); z = y W~^T + adapters(y); the loss of z V^T.  The binarized layer's real weights, the gain, the adapters and the head
all take a step of AdamW.
"""
import numpy as np
import pytest
import torch

from paper_1804_02941_amd import binding as dab

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
T, K, F, V, N, R = 192, 160, 96, 500, 3, 8


class Block:
    """Everything that a step reads and writes; fp32 throughout, so that it can be held to float64 closely."""

    def __init__(self, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)

        def normal(*shape, by=1.0):
            return by * torch.randn(shape, generator=g, device=DEV)
        self.x, self.r, self.gain = normal(T, K), normal(T, K), 1 + normal(K, by=0.1)
        self.W, self.V = normal(F, K, by=K ** -0.5), normal(V, F, by=F ** -0.5)
        self.A, self.B, self.scale = normal(N, R, K, by=K ** -0.5), normal(N, R, F, by=0.1), 0.5 + torch.rand(N, generator=g, device=DEV)
        self.ids = torch.randint(-1, N, (T // 16,), generator=g, device=DEV).repeat_interleave(16).int()
        self.words = torch.randint(0, V, (T,), generator=g, device=DEV)
        self.words[::11] = -100
        self.live = self.words != -100
        self.weight = self.live.float() / self.live.sum()
        self.grads = {k: torch.zeros_like(getattr(self, k)) for k in ("W", "gain", "A", "B", "V")}
        self.states = {k: dab.adamw_states(getattr(self, k), 8 if k in ("A", "V") else 32) for k in self.grads}
        self.count = torch.zeros(1, dtype=torch.int64, device=DEV)
        self.jobs = dab.adamw_jobs([{"P": getattr(self, k), "G": self.grads[k], "M": self.states[k][0], "V": self.states[k][1],
                                     "weight_decay": 0.0 if k == "gain" else 0.01} for k in self.grads])

    def binarized(self):
        centred = dab.dab_mean_center_clamp(self.W.view(F, K, 1, 1)).view(F, K)
        est = dab.dab_estimate_alpha_beta(centred)
        E, _ = dab.dab_pack_weights(centred.view(F, K, 1, 1), est["thr_val"], est["thr_idx"], est["alpha_is_upper"])
        return centred, est, E

    def step(self):
        """Forward, backward, and a step; what a test looks at."""
        centred, est, E = self.binarized()
        y, h, rstd, saved = dab.dab_rms_norm(self.x, self.gain, residual=self.r, save=True)
        base = dab.dab_wbin_fc(y, E, est["alpha"], est["beta"])
        z, U = dab.dab_adapters(y, self.ids, self.A, self.B, self.scale, base=base)
        loss, lse = dab.dab_head_loss(z, self.V, self.words)
        dz, dV = dab.dab_head_loss_gradient(z, self.V, self.words, lse, self.weight)
        Wt = dab.dab_binarized_weights(centred, est["alpha"], est["beta"], est["thr_val"], est["thr_idx"], est["alpha_is_upper"])
        dy, dA, dB = dab.dab_adapters_gradient(dz, y, U, self.ids, self.A, self.B, self.scale, base=dz @ Wt)
        dx, dgain = dab.dab_rms_norm_gradient(dy, h, self.gain, rstd)
        dWt = dab.dab_ckpt8_weight_gradient(dz, *saved, K)
        dW = dab.dab_weight_gradient(centred, est["thr_val"], est["thr_idx"], est["alpha_is_upper"], upstream=dWt)
        for k, v in (("W", dW), ("gain", dgain), ("A", dA), ("B", dB), ("V", dV)):
            self.grads[k].copy_(v)
        self.count.add_(1)
        dab.dab_adamw(self.jobs, 1e-2, self.count, seed=5)
        return {"loss": loss, "dx": dx, "dWt": dWt, "Wt": Wt, "z": z, "saved": dab.dab_ckpt8_restore(*saved, K), **{"d" + k: v.clone() for k, v in self.grads.items()}}


def test_gradients_of_the_whole_step():
    b = Block()
    before = {k: getattr(b, k).double().cpu() for k in ("x", "r", "gain", "A", "B", "V", "scale")}
    got = b.step()
    x, r, gain, A, B, Vw, scale = (before[k].requires_grad_() for k in ("x", "r", "gain", "A", "B", "V", "scale"))
    Wt = got["Wt"].double().cpu().requires_grad_()
    h = x + r
    y = h / torch.sqrt((h * h).mean(dim=1, keepdim=True) + 1e-5) * gain
    ids = b.ids.cpu()
    z = y @ Wt.t()
    rows = []
    for t in range(T):
        i = int(ids[t])
        rows.append(z[t] + (scale[i] * ((A[i] @ y[t]) @ B[i]) if i >= 0 else 0))
    z = torch.stack(rows)
    logits = z @ Vw.t()
    words, live = b.words.cpu(), b.live.cpu()
    loss = torch.logsumexp(logits, 1) - logits.gather(1, torch.where(live, words, 0).unsqueeze(1)).squeeze(1)
    ((loss * live).sum() / live.sum()).backward()
    # Sums of up to some 500 terms in fp32, in chains of five products: 5 * 500 * 2^-24 = 1.5e-4 of the sums of magnitudes, which are some ten times the
    # results at the most: held to 2e-3 of the largest.
    def near(a, w, by=2e-3):
        a, w = a.double().cpu(), w.detach()
        assert float((a - w).abs().max()) <= by * float(w.abs().max())
    near(got["loss"], loss * live)
    near(got["z"], z)
    for k, w in (("dx", x.grad), ("dgain", gain.grad), ("dA", A.grad), ("dB", B.grad), ("dV", Vw.grad)):
        near(got[k], w)
    assert torch.equal(x.grad, r.grad)
    # the layer's weights see its input in 8 bits, off by at most 1/127 of a group's largest value
    near(got["saved"], y, by=1 / 127)
    near(got["dWt"], Wt.grad, by=0.02)


def test_steps_move_everything_and_are_the_same_every_time():
    a, b = Block(1), Block(1)
    for _ in range(3):
        p, q = a.step(), b.step()
        assert all(torch.equal(p[k], q[k]) for k in p)
    for k in a.grads:
        assert torch.equal(getattr(a, k), getattr(b, k)) and not torch.equal(getattr(a, k), getattr(Block(1), k)) and bool(getattr(a, k).isfinite().all())


def test_a_captured_step_is_the_eager_one():
    a, b = Block(2), Block(2)
    a.step(), b.step()                                             # (the caches of libraries and the allocator are warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = a.step()
    for i in range(4):
        for t in (a, b):
            t.x.normal_(generator=torch.Generator(device=DEV).manual_seed(i))
        graph.replay()
        want = b.step()
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(out[k], want[k]), (i, k)
        for k in a.grads:
            assert torch.equal(getattr(a, k), getattr(b, k)), (i, k)


def test_what_was_trained_is_served():
    b = Block(3)
    for _ in range(2):
        b.step()
    y, _, _, _ = dab.dab_rms_norm(b.x, b.gain, residual=b.r)
    Q, S = dab.dab_w4_pack(b.W)
    W4 = dab.dab_w4_unpack(Q, S, F, K).double().cpu().numpy()
    many = dab.dab_w4_adapters(y, Q, S, F, b.ids, b.A, b.B, b.scale)
    beside, _ = dab.dab_adapters(y, b.ids, b.A, b.B, b.scale, base=dab.dab_w4_matvec(y, Q, S, F))
    y64, A, B, s = (t.double().cpu().numpy() for t in (y, b.A, b.B, b.scale))
    for t in range(0, T, 7):
        i = int(b.ids[t])
        one = dab.dab_w4_adapters(y[t:t + 1], Q, S, F, b.ids[t:t + 1], b.A, b.B, b.scale)[0].double().cpu().numpy()
        want = W4 @ y64[t] + (s[i] * ((A[i] @ y64[t]) @ B[i]) if i >= 0 else 0)
        size = np.abs(W4) @ np.abs(y64[t]) + (s[i] * ((np.abs(A[i]) @ np.abs(y64[t])) @ np.abs(B[i])) if i >= 0 else 0)
        off = (3 * K + R + 10) * 2.0 ** -24 * size
        for got in (one, many[t].double().cpu().numpy(), beside[t].double().cpu().numpy()):
            assert np.all(np.abs(got - want) <= off)
