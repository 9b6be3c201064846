"""The factor of a branch, alpha over the probability of being kept, is one float: where it is infinite, and a kept zero would come out as NaN, the
residual block's calls are refused.  No GPU is needed."""
import ctypes

import pytest

from paper_2409_11902_amd import binding as B

MB = 1 << 20
LARGEST = 3.4028234e38


def codes(**over):
    """What the calls answer that check a descriptor and launch nothing."""
    L, n = B.lib(), ctypes.c_size_t()
    r = [L.cac_linear_workspace_size(B.make_linear_desc(40, 64, 48, **over), op, ctypes.byref(n)) for op in (0, 1)]
    return r + [L.cac_block_norm_workspace_size(B.make_block_norm_desc(40, 64, **over), op, ctypes.byref(n)) for op in (0, 1)]


@pytest.mark.parametrize("alpha,p", [(LARGEST, 0.5), (-LARGEST, 0.5), (LARGEST, 2.0 ** -16), (1e38, 0.9), (1e34, 1 - 2.0 ** -16)])
def test_infinite_factors(alpha, p):
    assert codes(alpha=alpha, p=p) == [-1] * 4
    assert b"alpha" in B.lib().cac_last_error()
    assert B.lib().cac_dropout(B.make_dropout_desc(40, 64, alpha=alpha, p=p), 64 * MB, None, 128 * MB, 192 * MB, None) == -1
    assert b"alpha" in B.lib().cac_last_error()


@pytest.mark.parametrize("alpha,p", [(LARGEST, 0.0), (-LARGEST, 1.0), (1.7e38, 0.5), (5e33, 1 - 2.0 ** -16), (0.0, 0.5), (1e-45, 0.1)])
def test_finite_factors(alpha, p):
    assert codes(alpha=alpha, p=p) == [B.CAC_OK] * 4
