"""Orthogonalised updates of narrow matrices are as near to the exact ones as float arithmetic's are.

Halves of a float lose 2^-23 of an operand where float loses 2^-24, and sums in steps of 16 terms are rounded a sixteenth as often as term by
term: the two are about even, and a fifth is allowed."""
import pytest
import torch

from paper_2409_11902_amd import binding as B
from test_gpu_muon import A_, B_, C_, DEV, orthogonal, rel, run

pytestmark = pytest.mark.gpu


def strong_and_weak(m, n, seed):
    """A few strong directions whose strength falls off, over noise: the weak ones' errors grow the most."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    r = min(m, n, 32)
    x = torch.randn(1, m, r, generator=g, device=DEV) * torch.exp(-0.15 * torch.arange(r, device=DEV))
    return x @ (torch.randn(1, r, n, generator=g, device=DEV) * 1e-3) + torch.randn(1, m, n, generator=g, device=DEV) * 2e-4


def in_floats(x):
    tall = x.shape[1] > x.shape[2]
    x = x.mT if tall else x
    x = x / (x.square().sum(dim=(-2, -1), keepdim=True).sqrt() + 1e-7)
    for _ in range(5):
        s = x @ x.mT
        x = A_ * x + (B_ * s + C_ * (s @ s)) @ x
    return x.mT if tall else x


@pytest.mark.parametrize("shape", [(64, 64), (64, 128), (64, 256), (50, 200), (64, 576), (576, 64), (64, 4096)])
def test_as_near_as_float_arithmetic(shape):
    here = plain = 0.0
    for seed in range(12):
        G = strong_and_weak(*shape, seed)
        want = orthogonal(G)
        here += rel(run(G, B.F32), want)
        plain += rel(in_floats(G), want)
    assert here <= 1.2 * plain, (here / 12, plain / 12)
