"""The example of adapters beside a 4-bit layer runs, and its gradients are those of its formula in float64."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_it_runs():
    import adapt_and_serve
    same = adapt_and_serve.main(steps=3)
    assert 0.0 <= same <= 1.0


def test_its_gradients():
    import adapt_and_serve as ex
    model = ex.Model(seed=2)
    model.B.normal_(generator=model.g).mul_(0.1)
    X, tasks, words = model.batch(96)
    loss = model.gradients(X, tasks, words)
    A, B, gain = (t.double().cpu().requires_grad_() for t in (model.A, model.B, model.gain))
    x, W, V, i = X.double().cpu(), model.W4.double().cpu(), model.V.double().cpu(), tasks.long().cpu()
    y = x / torch.sqrt((x * x).mean(dim=1, keepdim=True) + 1e-5) * gain
    u = (A[i] * y[:, None, :]).sum(dim=2)
    z = y @ W.t() + (u[:, :, None] * B[i]).sum(dim=1)
    want = torch.nn.functional.cross_entropy(z @ V.t(), words.cpu())
    want.backward()
    # chains of four products of up to 1000 terms in fp32: 4 * 1000 * 2^-24 = 2.4e-4 of sums of magnitudes, up to ten times their results
    assert abs(float(loss) - float(want.detach())) <= 1e-3 * float(want.detach())
    for got, w in ((model.grads["A"], A.grad), (model.grads["B"], B.grad), (model.grads["gain"], gain.grad)):
        assert float((got.double().cpu() - w).abs().max()) <= 3e-3 * float(w.abs().max())
