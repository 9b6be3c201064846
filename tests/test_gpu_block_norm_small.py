"""The ends of float's range, as the header has them.

Rows of numbers so small that their mean square is below the least normal float, without an epsilon to hide it, and rows of zeros with an epsilon that
is itself below it.

Tolerances.  Numbers are 2^-66 times small whole ones, ten of them 3 or -3 in each row of 40: a mean square is 2^-131 at least.  Squares, their sum and
its product with 1 / D are off by half a step of 2^-149 each on the average of their terms (rms: squares and sums are exact): 2 * 2^-150 of 2^-131, of which the root takes half.  With its
own roundings and the products' that is below 2^-18, the tolerance of the norms' other tests, of xhat.  A gradient, of a size of 2^66 g, meets it in each of the three parts of its
formula: 4 * 2^-18 of (1 + xhat^2) times the row's largest g.  Results are rounded to half a step."""
import pytest
import torch

from block_util import DEV, HALF, TYPES, close, norm, norm_back
from paper_2409_11902_amd import binding as B

pytestmark = pytest.mark.gpu
T, D, E = 9, 40, 2.0 ** -18


def rows(dtype):
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    x = torch.randint(-3, 4, (T, D), generator=g, device=DEV).float()
    x[:, 0:10:2], x[:, 1:10:2] = 3, -3
    return (x * 2.0 ** -66).to(TYPES[dtype])


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("kind", [B.NORM_RMS, B.NORM_LAYER])
def test_tiny_rows_without_epsilon(kind, dtype):
    F = rows(dtype)
    d = B.make_block_norm_desc(T, D, dtype=dtype, post=B.NORM_NONE, pre=kind, eps_pre=0.0)
    H, dS = torch.empty_like(F), torch.empty_like(F)
    B.cac_block_norm_fwd(d, F, None, None, None, None, None, None, None, None, H)
    want, xhat, inv, _ = norm(kind, F.double(), 0.0, None, None)
    assert bool(torch.isfinite(H).all())
    close("H", H, want, E * (1 + want.abs()) + HALF[dtype] * want.abs())
    g = torch.randn(T, D, device=DEV).to(TYPES[dtype])
    B.cac_block_norm_bwd(d, None, F, None, None, None, None, g, None, None, dS, None, None, None, None, None, None,
                         torch.empty(max(16, B.cac_block_norm_workspace_size(d, B.BLOCK_NORM_BWD)), dtype=torch.uint8, device=DEV))
    want = norm_back(kind, xhat, inv, g.double())
    top = g.double().abs().amax(1, keepdim=True) * (1 + xhat.square().amax(1, keepdim=True))
    assert bool(torch.isfinite(dS).all())
    close("dS", dS, want, 4 * E * inv * top + HALF[dtype] * want.abs())


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("kind", [B.NORM_RMS, B.NORM_LAYER])
def test_zeros_with_a_tiny_epsilon(kind, dtype):
    F, b = torch.zeros(T, D, device=DEV).to(TYPES[dtype]), torch.arange(D, device=DEV).float()
    d = B.make_block_norm_desc(T, D, dtype=dtype, post=B.NORM_NONE, pre=kind, eps_pre=1e-40)
    H = torch.empty_like(F)
    B.cac_block_norm_fwd(d, F, None, None, None, None, None, b, None, None, H)
    assert torch.equal(H.float(), b.expand(T, D))


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("kind", [B.NORM_RMS, B.NORM_LAYER])
@pytest.mark.parametrize("D", [40, 1001, 9000])
def test_rows_whose_squares_leave_the_range(D, kind, dtype):
    """Their xhat is 0: H is b, and no gradient comes through the norm."""
    F, b = torch.randn(T, D, device=DEV).mul_(1e25).to(TYPES[dtype]), torch.arange(D, device=DEV).float()
    d = B.make_block_norm_desc(T, D, dtype=dtype, post=B.NORM_NONE, pre=kind)
    H, dR, dH, dS = (torch.randn(T, D, device=DEV).to(TYPES[dtype]) for _ in range(4))
    B.cac_block_norm_fwd(d, F, None, None, None, None, None, b, None, None, H)
    assert torch.equal(H, b.expand(T, D).to(TYPES[dtype]))
    B.cac_block_norm_bwd(d, None, F, None, None, None, None, dH, dS, None, dR, None, None, None, None, None, None,
                         torch.empty(max(16, B.cac_block_norm_workspace_size(d, B.BLOCK_NORM_BWD)), dtype=torch.uint8, device=DEV))
    assert torch.equal(dR, dS)
