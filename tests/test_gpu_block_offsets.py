"""Tensors of more than 2^32 bytes and elements: the last rows of the residual block's operators, and the first, against their formulas.

Tolerances: those of the operators' own tests (dropout: 4 roundings of 2^-24 and half a step; a product of 16 terms: (4 sqrt 16 + 8) 2^-23 of the sum of
magnitudes and half a step; norms of 1024 columns: 2^-18 of a row's largest and half a step)."""
import numpy as np
import pytest
import torch

from block_util import DEV, close, norm, philox
from paper_2409_11902_amd import binding as B

pytestmark = pytest.mark.gpu
HALF = 2.0 ** -8
LOW = np.uint64(0xFFFFFFFF)


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def keep_of_rows(rows, cols, p, site, rng):
    t = int(p * 65536 + 0.5)
    across = -(-cols // 8)
    g = (np.asarray(rows, dtype=np.uint64)[:, None] * np.uint64(across) + np.arange(across, dtype=np.uint64)).ravel()
    one = np.ones_like(g)
    w = philox((g & LOW, (g >> np.uint64(32)) | np.uint64(site << 8), one * np.uint64(rng[1] & 0xFFFFFFFF), one * np.uint64(rng[1] >> 32)),
               (rng[0] & 0xFFFFFFFF, rng[0] >> 32))
    bits = np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], axis=1).reshape(len(rows), across * 8)[:, :cols]
    return torch.from_numpy((bits >= t).astype(np.float64)).to(DEV) * (65536 / (65536 - t))


def some(T):
    return [0, 1, T // 2, (1 << 31) // 1024 + 1, T - 2, T - 1]


def big(T, D, seed, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(T, D, dtype=torch.bfloat16, device=DEV).normal_(0.0, std, generator=g)


def test_dropout():
    T, D, rng = (1 << 22) + 5, 1024, (77, 3)
    x, r = big(T, D, 1), big(T, D, 2)
    y = torch.empty_like(x)
    B.cac_dropout(B.make_dropout_desc(T, D, p=0.25, site=9), x, r, torch.tensor(rng, device=DEV), y)
    at = some(T)
    part = x[at].double() * keep_of_rows(at, D, 0.25, 9, rng)
    want = part + r[at].double()
    close("Y", y[at], want, 4 * 2.0 ** -24 * (part.abs() + r[at].double().abs()) + HALF * want.abs())


def test_groups_past_32_bits():
    """Three groups of eight to each of 2^31 - 1 rows, in place."""
    T, D, rng = (1 << 31) - 1, 17, (5, 1)
    x = torch.ones(T, D, dtype=torch.bfloat16, device=DEV)
    B.cac_dropout(B.make_dropout_desc(T, D, p=0.5, site=2), x, None, torch.tensor(rng, device=DEV), x)
    at = [0, 1, 2, 3, (1 << 32) // 3 - 1, (1 << 32) // 3, (1 << 32) // 3 + 1, T - 3, T - 2, T - 1]
    assert torch.equal(torch.stack([x[k] for k in at]).double(), keep_of_rows(at, D, 0.5, 2, rng))


def test_linear():
    T, D, N, rng = (1 << 21) + 7, 16, 2056, (9, 2)
    X, W, dY = big(T, D, 3), big(N, D, 4, 0.25), big(T, N, 5)
    d = B.make_linear_desc(T, D, N, act=B.ACT_SILU, p=0.25, site=4)
    ws = torch.empty(max(B.cac_linear_workspace_size(d, op) for op in (0, 1)), dtype=torch.uint8, device=DEV)
    Y, dX, r = torch.empty_like(dY), torch.empty_like(X), torch.tensor(rng, device=DEV)
    B.cac_linear_fwd(d, X, W, None, None, r, Y, ws)
    B.cac_linear_bwd(d, X, W, None, dY, r, dX, None, None, ws)
    at = some(T)[:3] + [T - 2, T - 1]
    x, w = X[at].double(), W.double()
    keep, u = keep_of_rows(at, N, 0.25, 4, rng), x @ w.t()
    e_u = 24 * 2.0 ** -23 * (x.abs() @ w.abs().t())
    s = torch.sigmoid(u)
    close("Y", Y[at], keep * u * s, keep * (1.13 * e_u + 2.0 ** -20 * u.abs()) + (HALF + 2.0 ** -21) * (keep * u * s).abs())
    g = dY[at].double() * keep * s * (1 + u * (1 - s))
    e_g = dY[at].double().abs() * keep * (0.5 * e_u + 2.0 ** -20) + HALF * g.abs()
    want = g @ w
    close("dX", dX[at], want, e_g @ w.abs() + 2.0 ** -23 * (4 * N ** 0.5 + 8) * (g.abs() @ w.abs()) + HALF * want.abs())


def test_norms():
    T, D, rng = (1 << 22) + 3, 1024, (31, 8)
    F, R = big(T, D, 6), big(T, D, 7)
    d = B.make_block_norm_desc(T, D, post=B.NORM_RMS, pre=B.NORM_LAYER, p=0.25, site=6)
    S, H, r = torch.empty_like(F), torch.empty_like(F), torch.tensor(rng, device=DEV)
    B.cac_block_norm_fwd(d, F, R, None, None, None, None, None, r, S, H)
    at = some(T)
    n = norm(B.NORM_RMS, F[at].double(), 1e-5, None, None)[0]
    total = R[at].double() + keep_of_rows(at, D, 0.25, 6, rng) * n
    e = 2.0 ** -18 * (total.abs() + n.abs().amax(1, keepdim=True))
    close("S", S[at], total, e + HALF * total.abs())
    want = norm(B.NORM_LAYER, total, 1e-5, None, None)[0]
    close("H", H[at], want, 8 * e.amax(1, keepdim=True) * (1 + want.abs().amax(1, keepdim=True)) + HALF * want.abs())
    dR = R  # (in place of dS: what the forward pass had as R serves as a gradient)
    dS = R[at].double()
    ws = torch.empty(B.cac_block_norm_workspace_size(d, B.BLOCK_NORM_BWD), dtype=torch.uint8, device=DEV)
    dw = torch.empty(D, device=DEV)
    B.cac_block_norm_bwd(d, F, S, None, None, None, None, H, R, r, dR, None, None, dw, None, None, None, ws)
    _, xhat, inv, _ = norm(B.NORM_LAYER, S[at].double(), 1e-5, None, None)
    g = H[at].double()
    want = dS + inv * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    scale = dS.abs() + inv * g.abs().amax(1, keepdim=True) * (1 + xhat.abs().amax(1, keepdim=True) ** 2)
    close("dR", dR[at], want, 2.0 ** -16 * scale + HALF * want.abs())
    assert bool(torch.isfinite(dw).all())
