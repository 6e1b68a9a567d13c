"""The token model with the norm, the trained projection and inputs in 8 bits: gradients against automatic differentiation in float64, and that
it runs."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from oracle import tokens as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import token_experts
    return token_experts


def test_gradients_of_the_model_with_the_norm(example):
    """fp32: every gradient within 5e-5 of its largest element (sums of at most 300 terms through seven operators, each with a relative error
    below 1e-6; the margin is for the cancellation in them)."""
    m = example.Model(vocab=50, dim=24, experts=4, classes=30, tokens=150, p=0.25, seed=3, norm=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    m.gamma += 0.2 * torch.randn(24, generator=g, device="cuda")
    ids = m.batch()
    d = torch.randn(150, 30, generator=g, device="cuda")
    logits = m.forward(ids)
    m.backward(ids, d)
    keep = torch.from_numpy(T.dropout_keep(0, 150 * 24, 0.25, 3, 0).reshape(150, 24))
    f64 = lambda t: t.detach().double().cpu()  # noqa: E731
    table, W, Wout, router, gamma = (f64(t).requires_grad_() for t in (m.table, m.W, m.Wout, m.router, m.gamma))
    h = torch.where(keep, table[ids.cpu()] * m.scale * (65536.0 / (65536 - 16384)), torch.zeros((), dtype=torch.float64))
    u = gamma * h * (h.square().mean(1, keepdim=True) + example.EPS).rsqrt()
    choice = m.choice.cpu().long().view(150, 2)
    score = u @ router.T
    assert torch.equal(choice, score.topk(2, dim=1).indices)
    gate = score.gather(1, choice).softmax(1)
    y = torch.stack([torch.stack([W[choice[t, j]] @ u[t] for j in range(2)]) for t in range(150)])
    z = h + (gate[:, :, None] * y).sum(1)
    ref = z @ Wout.T
    (ref * f64(d)).sum().backward()
    for got, want in ((logits, ref), (m.dtable, table.grad), (m.dW, W.grad), (m.dWout, Wout.grad), (m.drouter, router.grad), (m.dgamma, gamma.grad)):
        want = want.detach()
        assert float((f64(got) - want).abs().max()) <= 5e-5 * float(want.abs().max())


@pytest.mark.parametrize("norm,kept", [(True, False), (False, True), (True, True)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_it_runs(example, dtype, norm, kept):
    losses = example.train(6, dtype=dtype, vocab=128, classes=128, dim=64, experts=4, tokens=1024, norm=norm, kept=kept)
    assert all(np.isfinite(losses))
    again = example.train(6, dtype=dtype, vocab=128, classes=128, dim=64, experts=4, tokens=1024, norm=norm, kept=kept)
    assert losses == again
