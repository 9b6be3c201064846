"""Sums over many rows: weights', biases' and gates' gradients against sums in 64 bits, taken over all rows, and rows' gradients beside them.

Tolerances.  Where a test of norms or of dense layers has formulas for them, those.  Of 2^21 rows and more the sums are compared in the 2-norm.  A float sum of n
terms of random signs, in p parts one after the other, is off by about 2^-25 of its partial sums at every step: sqrt(n / 2) 2^-25 times the sum's own size sqrt(n) over sqrt(p), 3e-6 of
it at n / p = 2^13, and by what its terms are off by, 2^-22 each of random signs: 1e-5 of all.  A row that is left out or comes in twice changes it by
1 / sqrt(T) in the mean, 5e-4.  bfloat16: the result's rounding and dU's, 2^-8 as in the dense layer's tests."""
import pytest
import torch

import test_gpu_block_norm as norms
import test_gpu_linear as linears
from block_util import DEV, act, norm, norm_back, rel
from test_gpu_block_offsets import big

from paper_2409_11902_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("T,D,gate_rows", [(200003, 24, 0), (200003, 24, 200003), (100001, 136, 49), (100001, 129, 20000), (300000, 16, 3), (40001, 520, 13000), (6007, 8200, 0)])
def test_norms(T, D, gate_rows, dtype):
    norms.check(norms.make(T, D, dtype, B.NORM_LAYER, B.NORM_LAYER, gate_rows=gate_rows, p=0.1 if D < 1000 else 0.0, alpha=0.7))


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape,kind", [((200003, 24, 40), B.ACT_GELU), ((131073, 8, 264), B.ACT_NONE), ((100001, 33, 7), B.ACT_RELU)])
def test_dense_layers(shape, kind, dtype):
    linears.check(linears.make(*shape, dtype, kind, p=0.1))


def chunks(T):
    return [slice(k, min(T, k + (1 << 17))) for k in range(0, T, 1 << 17)]


@pytest.mark.parametrize("gate_rows", [0, 1 << 20])
def test_norms_of_four_million_rows(gate_rows):
    T, D = (1 << 22) + 3, 1024
    F, S, dH = big(T, D, 1), big(T, D, 2), big(T, D, 3)
    d = B.make_block_norm_desc(T, D, post=B.NORM_LAYER, pre=B.NORM_RMS, gate_rows=gate_rows)
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    w_post, b_post, w_pre = (torch.randn(D, generator=g, device=DEV) * 0.3 + 1 for _ in range(3))
    G = -(-T // gate_rows) if gate_rows else 1
    gate = torch.randn(G, D, generator=g, device=DEV) if gate_rows else None
    dR, dF, got = torch.empty_like(F), torch.empty_like(F), {k: torch.empty(D, device=DEV) for k in ("w_post", "b_post", "w_pre", "b_pre")}
    dgate = torch.empty_like(gate) if gate_rows else None
    ws = torch.empty(B.cac_block_norm_workspace_size(d, B.BLOCK_NORM_BWD), dtype=torch.uint8, device=DEV)
    B.cac_block_norm_bwd(d, F, S, gate, w_post, b_post, w_pre, dH, None, None, dR, dF, dgate, got["w_post"], got["b_post"], got["w_pre"], got["b_pre"], ws)
    want = {k: torch.zeros(D, dtype=torch.float64, device=DEV) for k in got}
    want_gate = torch.zeros(G, D, dtype=torch.float64, device=DEV)
    for c in chunks(T):
        dh = dH[c].double()
        _, shat, sinv, _ = norm(B.NORM_RMS, S[c].double(), 1e-5, None, None)
        n, fhat, finv, _ = norm(B.NORM_LAYER, F[c].double(), 1e-5, w_post, b_post)
        a = norm_back(B.NORM_RMS, shat, sinv, dh * w_pre.double())
        at = c.start // gate_rows if gate_rows else 0  # (a chunk's rows have one gate)
        dn = a * gate[at].double() if gate_rows else a
        for k, v in (("w_post", dn * fhat), ("b_post", dn), ("w_pre", dh * shat), ("b_pre", dh)):
            want[k] += v.sum(0)
        if gate_rows:
            want_gate[at] += (a * n).sum(0)
        rows = norm_back(B.NORM_LAYER, fhat, finv, dn * w_post.double())
        assert rel(dR[c], a) <= 2.0 ** -8 and rel(dF[c], rows) <= 2.0 ** -8
    for k in got:
        assert rel(got[k], want[k]) <= 1e-5, (k, rel(got[k], want[k]))
    if gate_rows:
        assert rel(dgate[:-1], want_gate[:-1]) <= 1e-5 and rel(dgate[-1], want_gate[-1]) <= 1e-5


@pytest.mark.parametrize("kind", [B.ACT_SILU, B.ACT_NONE])
def test_a_dense_layer_of_two_million_rows(kind):
    T, D, N = (1 << 21) + 7, 16, 2056
    X, W, dY = big(T, D, 3), big(N, D, 4, 0.25), big(T, N, 5)
    b = torch.randn(N, device=DEV).bfloat16()
    d = B.make_linear_desc(T, D, N, has_bias=1, act=kind)
    ws = torch.empty(max(16, B.cac_linear_workspace_size(d, B.LINEAR_BWD)), dtype=torch.uint8, device=DEV)
    dX, dW, db = torch.empty_like(X), torch.empty_like(W), torch.empty_like(b)
    B.cac_linear_bwd(d, X, W, b, dY, None, dX, dW, db, ws)
    w, want_w, want_b = W.double(), torch.zeros(N, D, dtype=torch.float64, device=DEV), torch.zeros(N, dtype=torch.float64, device=DEV)
    for c in chunks(T):
        x = X[c].double()
        g = dY[c].double()
        if kind != B.ACT_NONE:
            g = g * act(kind, x @ w.t() + b.double())[1]
        want_w += g.t().contiguous() @ x
        want_b += g.sum(0)
        assert rel(dX[c], g @ w) <= 2.0 ** -8
    assert rel(dW, want_w) <= 2.0 ** -8 and rel(db, want_b) <= 2.0 ** -8, (rel(dW, want_w), rel(db, want_b))
