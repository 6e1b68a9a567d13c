"""The token and expert layers together: gradients of a whole model against automatic differentiation in float64, and training."""
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


def test_gradients_of_the_model(example):
    """fp32: every gradient within 2e-5 of its largest element (sums of at most 300 terms through four layers, each with a relative
    error below 1e-6; the margin is for the cancellation in them)."""
    m = example.Model(vocab=50, dim=24, experts=4, classes=30, tokens=150, p=0.25, seed=3)
    ids = m.batch()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    d = torch.randn(150, 30, generator=g, device="cuda")
    logits = m.forward(ids)
    m.backward(ids, d)
    keep = torch.from_numpy(T.dropout_keep(0, 150 * 24, 0.25, 3, 0).reshape(150, 24))
    f64 = lambda t: t.detach().double().cpu()  # noqa: E731
    table, W, Wout = (f64(t).requires_grad_() for t in (m.table, m.W, m.Wout))
    h = torch.where(keep, table[ids.cpu()] * m.scale * (65536.0 / (65536 - 16384)), torch.zeros((), dtype=torch.float64))
    choice, gate = m.choice.cpu().long().view(150, 2), f64(m.gate)
    y = torch.stack([torch.stack([W[choice[t, j]] @ h[t] for j in range(2)]) for t in range(150)])
    z = h + (gate[:, :, None] * y).sum(1)
    ref = z @ Wout.T
    (ref * f64(d)).sum().backward()
    for got, want in ((logits, ref), (m.dtable, table.grad), (m.dW, W.grad), (m.dWout, Wout.grad)):
        want = want.detach()
        assert float((f64(got) - want).abs().max()) <= 2e-5 * float(want.abs().max())
    counts = np.bincount(ids.cpu().numpy(), minlength=50)
    assert np.allclose(f64(m.A_table).numpy(), counts / 150, rtol=1e-6, atol=0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training(example, dtype):
    losses = example.train(15, dtype=dtype, vocab=128, classes=128, dim=64, experts=4, tokens=1024)
    assert all(np.isfinite(losses))
    assert losses[-1] < 0.5 * losses[0]


def test_training_repeats_bit_for_bit(example):
    a, b = (example.train(4, vocab=100, classes=60, dim=40, experts=3, tokens=700) for _ in range(2))
    assert a == b
