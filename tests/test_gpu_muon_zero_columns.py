"""Orthogonalised updates of narrow matrices some of whose columns are zeros, as a filter's gradient has where an input channel is dead.

The tolerance is that of the other orthogonalised updates: three times what float arithmetic ends at on such inputs."""
import pytest
import torch

from paper_2409_11902_amd import binding as B
from test_gpu_muon import TOL, gradient, orthogonal, rel, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1.0, 1e-12, 1e-20, 1e-25, 1e-30])
@pytest.mark.parametrize("shape", [(2, 64, 300), (2, 300, 64), (2, 64, 1100), (1, 33, 8192), (2, 8192, 20)])
@pytest.mark.parametrize("where", ["first", "middle", "last"])
def test_columns_of_zeros_do_not_set_the_scale(shape, where, scale):
    G = gradient(*shape, "gaussian", seed=3)
    x = G if shape[1] < shape[2] else G.mT                      # (its long side last)
    n = x.shape[2]
    # 256 and more whole columns, and some on either side of them: workgroups own up to 256 neighbours
    runs = {"first": (0, 260), "middle": (n // 4, min(n - 40, n // 4 + 600)), "last": (n - 270, n)}
    if n < 600:
        runs = {"first": (0, 130), "middle": (120, 260), "last": (250, 300)}
    a, b = runs[where]
    x[:, :, a:b] = 0
    G = G * scale
    got, want = run(G, B.F32), orthogonal(G)
    # (results of the smallest scales are below float's normal numbers when squared: compared as multiples of the scale)
    assert rel(got.double() / float(want.norm()), want / want.norm()) <= TOL[B.F32]


def test_columns_of_one_matrix_are_zeros_and_of_another_are_not():
    G = gradient(3, 64, 520, "falling", seed=5) * 1e-28
    G[0, :, :260] = 0
    G[2] = 0
    got, want = run(G, B.F32), orthogonal(G)
    for k in (0, 1):
        assert rel(got[k].double() / float(want[k].norm()), want[k] / want[k].norm()) <= TOL[B.F32]
    assert bool((got[2] == 0).all())
