"""The residual block's operators together, as examples/residual_step.py uses them: gradients of the whole step against automatic differentiation of
the formulas in 64 bits, and a captured step.

Tolerances.  Float: every call is within 1e-5 of its formula in the 2-norm; a gradient passes through seven of them, whose derivatives multiply such an
error by no more than about 3 each on these inputs' scales, and most of which meet it once: 1e-4.  bfloat16: up to nine roundings of tensors of a
spread of 2^-9 each on a gradient's way (five forward, h, a, f, s and out, and dout, df, da and dh), some through two ways: 9 * 2^-9 * sqrt 2 = 2.5e-2."""
import os
import sys

import pytest
import torch

from block_util import DEV, keep_factor
from paper_2409_11902_amd import binding as B

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))
pytestmark = pytest.mark.gpu
TOL = {B.F32: 1e-4, B.BF16: 2.5e-2}


def reference(block, X, labels):
    rows, width, hidden, _ = block.shape
    rng = block.rng.tolist()
    keep = {s: keep_factor(rows, n, p, s, rng).to(DEV) for s, n, p in ((1, hidden, block.wide.drop_p), (2, width, block.join.drop_p))}
    w = {k: v.double().requires_grad_() for k, v in block.w.items()}
    x = X.double().requires_grad_()

    def rms(v, weight, eps=1e-5):
        return v * (v.square().mean(1, keepdim=True) + eps).rsqrt() * weight

    u = rms(x, w["in"]) @ w["wide"].t() + w["wide_b"]
    a = keep[1] * u * 0.5 * torch.special.erfc(-u * 0.5 ** 0.5)
    f = a @ w["narrow"].t() + w["narrow_b"]
    s = x + block.join.alpha * keep[2] * w["gate"] * rms(f, w["post"])
    c = s - s.mean(1, keepdim=True)
    out = c * (c.square().mean(1, keepdim=True) + 1e-5).rsqrt() * w["pre"] + w["pre_b"]
    z = out @ w["head"].t()
    losses = torch.logsumexp(z, 1) - z.gather(1, labels[:, None]).squeeze(1)
    losses.mean().backward()
    return losses.detach(), {k: v.grad for k, v in w.items()}, x.grad


def rel(a, b):
    return float((a.double() - b).norm() / b.norm())


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("sizes", [dict(rows=256, width=192, hidden=512, classes=100), dict(rows=37, width=101, hidden=203, classes=50),
                                   dict(rows=1, width=64, hidden=128, classes=10), dict(rows=16, width=520, hidden=1040, classes=1000)])
def test_gradients_of_the_step(sizes, dtype):
    from residual_step import Block
    block = Block(dtype=dtype, seed=3, **sizes)
    block.rng[1] = 7
    X, labels = block.batch()
    block.forward(X, labels)
    block.backward(X, labels)
    losses, grads, dx = reference(block, X, labels)
    assert rel(block.losses, losses) <= TOL[dtype]
    for k, g in grads.items():
        assert rel(block.grad[k], g) <= TOL[dtype], (k, rel(block.grad[k], g))
    assert rel(block.dx, dx) <= TOL[dtype], rel(block.dx, dx)


def test_a_captured_step_draws_new_masks():
    """Replays follow an eager block that was made alike, bit for bit."""
    from residual_step import Block
    one, two = (Block(seed=5, rows=64, width=96, hidden=256, classes=40) for _ in range(2))
    X, labels = one.batch()
    one.step(X, labels)
    two.step(X, labels)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.step(X, labels)
    seen = []
    for _ in range(4):
        graph.replay()
        two.step(X, labels)
        torch.cuda.synchronize()
        assert torch.equal(one.losses, two.losses) and all(torch.equal(one.w[k], two.w[k]) for k in one.w)
        assert torch.equal(one.rng, two.rng)
        seen.append(one.a.clone())
    assert not torch.equal(seen[0] == 0, seen[1] == 0)


def test_the_example_runs():
    from residual_step import main
    history = main(steps=3, rows=64, width=64, hidden=128, classes=20)
    assert len(history) == 3 and all(h == h and h < float("inf") for h in history)
