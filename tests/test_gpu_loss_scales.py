"""The classifier's loss with operands and rows' gradients whose scales lie far apart.

The tolerance is that of the loss's float gradients elsewhere: sums of products of 22 bits and more."""
import pytest

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
