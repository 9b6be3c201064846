"""The classifier's loss with operands and rows' gradients whose scales lie far apart.

The tolerance is that of the loss's float gradients elsewhere: sums of products of 22 bits and more."""
import pytest
import torch

from paper_2409_11902_amd import binding as B
from test_gpu_loss import make, reference, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [100, 200, 1500])
def test_results_far_from_one_keep_their_bits(T):
    """Results that are normal numbers of float, of operands and rows' gradients whose scales lie far apart."""
    for scale_h, scale_w, scale_g in ((1e-30, 1.0, 1e-4), (1e-20, 1.0, 1e-14), (1e-25, 1e20, 1e-8), (1e25, 1e-25, 1e-10), (1e-20, 1e10, 1e20), (1.0, 1e-20, 1e-14)):
        t = make(T, 128, 300, B.F32, seed=5)
        t["H"] *= scale_h
        t["W"] *= scale_w
        t["gloss"] *= scale_g
        got, want = run(t), reference(t)
        for k, s in (("dW", scale_h * scale_g), ("dH", scale_w * scale_g), ("db", scale_g)):
            a, b = got[k].double() / s, want[k] / s
            assert float((a - b).norm() / b.norm()) <= 2e-5, (k, scale_h, scale_w, scale_g)


@pytest.mark.parametrize("large", [2.0 ** 10, 2.0 ** 20, 2.0 ** 30])
def test_operands_beside_a_large_one(large):
    """Numbers of H and W are off by 2^-24 of themselves and, held as two halves, by 2^-38 of their matrix's largest."""
    t = make(200, 512, 20000, B.F32, seed=6)
    t["H"][7] *= large
    t["W"][11] *= large
    t["labels"] = torch.where(t["labels"] == 11, 12, t["labels"])
    t["b"][11] = -torch.inf
    got, want = run(t), reference(t)
    h, w = t["H"].double().abs(), t["W"].double().abs()
    rows = torch.arange(200, device=h.device) != 7
    classes = torch.arange(20000, device=h.device) != 11
    z = 2.0 ** -38 * (h.max() * w[classes].sum(1).max() + w.max() * h[rows].sum(1).max())   # a logit's error for the halves
    z = float(z) + 2.0 ** -23 * 8 * float((h[rows] @ w[classes].t()).max())                  # ... and float's
    for k in ("loss", "lse"):
        assert float((got[k].double() - want[k])[rows].abs().max()) <= 2 * z + 2.0 ** -22 * float(want[k][rows].abs().max()), k
