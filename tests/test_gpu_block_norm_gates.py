"""Gradients of norms with many gates on the GPU, on both sides of the choice between slots that have whole gates' rows and workgroups that share one out, and
in more rounds of workgroups than one.  Formulas and tolerances are those of the norms' other tests."""
import pytest

from test_gpu_block_norm import check, make

from paper_2409_11902_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("D,rows,gates", [(2048, 8, 255), (2048, 8, 256), (2048, 8, 257), (2047, 49, 100), (4608, 12, 127), (4608, 12, 128), (4608, 12, 129), (512, 40, 513),
                                          (128, 49, 257), (40, 33, 300), (1024, 2, 256), (12000, 8, 127), (12000, 8, 128), (9001, 5, 129)])
def test_gates(D, rows, gates, dtype):
    """The last gate has two rows less than the others, or one row."""
    check(make(max(rows * gates - 2, rows * (gates - 1) + 1), D, dtype, B.NORM_LAYER, B.NORM_RMS, gate_rows=rows, p=0.1, alpha=0.7))
