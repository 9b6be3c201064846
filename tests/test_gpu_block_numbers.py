"""Tests of the residual block that compare element by element alone, once more with a comparison that NaN does not pass: an error that is no number is
no error below its bound."""
import pytest
import torch

import test_gpu_block_norm as norms
import test_gpu_block_offsets as offsets
import test_gpu_dropout as dropouts
import test_gpu_linear as linears
from paper_2409_11902_amd import binding as B

pytestmark = pytest.mark.gpu


def close(name, got, want, bound):
    err = (got.double() - want).abs()
    within = err <= bound
    assert bool(within.all()), f"{name}: {int((~within).sum())} of {err.numel()} off, {int(torch.isnan(err).sum())} of them no numbers"


@pytest.fixture(autouse=True)
def strict(monkeypatch):
    for module in (norms, offsets, dropouts, linears):
        monkeypatch.setattr(module, "close", close)
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_norms_of_special_rows_and_alone(dtype):
    norms.test_rows_of_one_number_zeros_infinities_and_nan(dtype)
    norms.test_a_norm_alone(dtype)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("post,pre", [(0, 1), (2, 2), (1, 2)])
def test_rows_of_one_column(post, pre, dtype):
    norms.test_norms(shape=(1, 1), post=post, pre=pre, dtype=dtype)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape", [(1, 1), (1, 9), (33, 1001), (1031, 520)])
def test_dropout(shape, dtype):
    dropouts.test_dropout(shape=shape, dtype=dtype, p=0.1)


@pytest.mark.parametrize("kind", [B.ACT_RELU, B.ACT_GELU, B.ACT_SILU])
def test_activations_at_their_ends(kind):
    linears.test_activations_at_their_ends(kind)


@pytest.mark.parametrize("test", [offsets.test_dropout, offsets.test_linear, offsets.test_norms], ids=["dropout", "linear", "norms"])
def test_large_tensors(test):
    test()
