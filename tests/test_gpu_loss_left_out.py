"""Rows that are left out of the classifier's loss have a gradient of 0, whatever stands in the weights."""
import pytest
import torch

from paper_2409_11902_amd import binding as B
from test_gpu_loss import make, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("big", [False, True])
@pytest.mark.parametrize("T", [5, 40, 64, 100, 500])
def test_rows_left_out_have_no_gradient_whatever_the_weights_hold(T, big, dtype):
    """dH of a row that is left out is 0 where W holds infinities and NaN, however few rows there are."""
    D, V = (200, 20000) if big else (136, 300)
    t = make(T, D, V, dtype, out=0.4, seed=T)
    t["labels"][1] = 7
    t["labels"][0] = -1
    t["W"][5, 3], t["W"][11, 64], t["W"][V - 1, D - 1] = torch.nan, torch.inf, -torch.inf
    gone = t["labels"] < 0
    got = run(t)
    assert bool((got["dH"][gone] == 0).all())
    assert bool((got["loss"][gone] == 0).all()) and bool((got["lse"][gone] == 0).all())
    assert bool(torch.isnan(got["dH"][~gone]).any())


def test_rows_left_out_have_no_gradient_in_pieces_of_the_classes():
    for dtype in (B.F32, B.BF16):
        t = make(20, 32, 600000, dtype, out=0.4, seed=1)
        t["labels"][1] = 7
        t["W"][5, 3], t["W"][599999, 31] = torch.nan, torch.inf
        gone = t["labels"] < 0
        assert bool((run(t)["dH"][gone] == 0).all())
