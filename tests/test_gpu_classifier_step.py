"""The example's training step on the GPU: the loss falls, and one step's numbers are those of plain operations."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.fixture()
def example():
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import classifier_step
        yield classifier_step
    finally:
        sys.path.pop(0)


def test_loss_falls(example):
    history = example.main(steps=40, classes=100)
    assert abs(history[0] - 4.6) < 1.0                      # near log 100 before anything is learnt
    assert sum(history[-5:]) / 5 < 0.5 * history[0]


def test_step_without_pooling_is_the_textbook_step(example):
    """With tiles of one pixel nothing is compressed: every updated parameter is that of plain automatic differentiation."""
    net = example.Network(images=24, channels=8, filters=32, side=8, classes=50, pool=1, seed=3)
    X, labels = net.batch()
    W, head, bias = (v.double().requires_grad_() for v in (net.W, net.head, net.bias))
    gamma, beta = net.gamma.double().requires_grad_(), net.beta.double().requires_grad_()
    cols = torch.nn.functional.unfold(X.double(), 3, padding=1)                     # [N, C * 9, pixels]
    y = (W.reshape(32, -1) @ cols).reshape(24, 32, 8, 8)
    mean, var = y.mean(dim=(0, 2, 3), keepdim=True), y.var(dim=(0, 2, 3), unbiased=False, keepdim=True)
    act = ((y - mean) * (var + 1e-5).rsqrt() * gamma.reshape(1, -1, 1, 1) + beta.reshape(1, -1, 1, 1)).relu()
    z = act.mean(dim=(2, 3)) @ head.t() + bias
    loss = torch.logsumexp(z, 1) - z.gather(1, labels[:, None]).squeeze(1)
    loss.mean().backward()

    def orthogonal(g):
        tall = g.shape[0] > g.shape[1]
        x = g.t() if tall else g
        x = x / (x.norm() + 1e-7)
        for _ in range(5):
            s = x @ x.t()
            x = 3.4445 * x + (-4.7750 * s + 2.0315 * s @ s) @ x
        return x.t() if tall else x

    with torch.no_grad():
        # the first step's nesterov momentum is a multiple of the gradient
        want = {"W": W - 0.02 * orthogonal(W.grad.reshape(32, -1)).reshape(W.shape),
                "head": head - 0.02 * (50 / 32) ** 0.5 * orthogonal(head.grad), "bias": bias - 0.02 * bias.grad,
                "gamma": gamma - 0.02 * gamma.grad, "beta": beta - 0.02 * beta.grad}
    got = net.step(X, labels)
    assert float((got.double() - loss.detach()).abs().max()) < 1e-4
    for name, w in want.items():
        assert float((getattr(net, name).double() - w).norm() / w.norm()) < 1e-4, name
