"""Orthogonalised updates and the optimiser's step made of them on the GPU, against Newton-Schulz products in 64 bits.

Tolerances.  Products keep 22 bits or more and sums are float, so a step's relative error is of the size of float
arithmetic's; an error of a direction that the gradient has little of grows by up to 3.4445 a step, 485 in five, while the
result's norm is that of the directions that it has much of.  Float arithmetic itself ends at up to 1.3e-5 on such inputs
(gaussian and falling spectra, sides to 4608); 4e-5 allows three times that.  A bfloat16 result adds one rounding, 2^-9 at most."""
import pytest
import torch

from paper_2409_11902_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
A_, B_, C_ = 3.4445, -4.7750, 2.0315
TOL = {B.F32: 4e-5, B.BF16: 2.0 ** -8}
TYPES = {B.F32: torch.float32, B.BF16: torch.bfloat16}


def gradient(batch, m, n, kind, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    x = torch.randn(batch, m, n, generator=g, device=DEV)
    if kind == "falling":
        r = min(m, n, 24)
        x = (torch.randn(batch, m, r, generator=g, device=DEV) * torch.exp(-0.2 * torch.arange(r, device=DEV))) @ torch.randn(
            batch, r, n, generator=g, device=DEV) + 0.2 * x
    return x * 1e-3


def orthogonal(x, steps=5):
    x = x.double()
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.mT
    x = x / (x.square().sum(dim=(-2, -1), keepdim=True).sqrt() + 1e-7)
    for _ in range(steps):
        s = x @ x.mT
        x = A_ * x + (B_ * s + C_ * (s @ s)) @ x
    return x.mT if tall else x


def call(d, op, *tensors, hyper=()):
    n = B.cac_muon_workspace_size(d, op)
    raw = torch.full((max(16, n) + 256,), 0xA5, dtype=torch.uint8, device=DEV)
    ws = raw[:max(16, n)]
    (B.cac_orthogonalise if op == B.MUON_ORTHOGONALISE else B.cac_muon_step)(d, *tensors, *hyper, ws)
    torch.cuda.synchronize()
    assert bool((raw[max(16, n):] == 0xA5).all()), "a write past the workspace"


def run(G, dtype, steps=5):
    from gpu_util import Guarded
    O = Guarded(G.shape, TYPES[dtype])
    d = B.make_muon_desc(G.shape[1], G.shape[2], batch=G.shape[0], dtype=dtype,
                         grad_dtype=B.F32 if G.dtype == torch.float32 else B.BF16, steps=steps)
    call(d, B.MUON_ORTHOGONALISE, G, O.t)
    O.check("O")
    return O.t


def rel(a, b):
    return float((a.double() - b).norm() / b.norm())


SHAPES = [
    (1, 1, 1), (1, 1, 9), (2, 5, 1), (1, 3, 5), (2, 17, 40), (3, 64, 64), (2, 64, 65), (2, 64, 128), (1, 40, 129), (2, 200, 64), (2, 64, 256),
    (1, 257, 33), (4, 64, 576), (2, 1001, 50), (1, 64, 2049), (1, 33, 8192), (1, 64, 8200), (2, 12000, 20), (1, 64, 16384), (1, 64, 16400), (2, 65, 65), (1, 100, 300), (3, 130, 67),
    (1, 129, 1152), (2, 300, 700), (3, 512, 512), (1, 1000, 513), (1, 700, 2049), (1, 2048, 256), (1, 1030, 1030),
]


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape", SHAPES)
def test_orthogonalised(shape, dtype):
    for kind in ("gaussian", "falling"):
        G = gradient(*shape, kind, seed=sum(shape))
        assert rel(run(G, dtype), orthogonal(G)) <= TOL[dtype], kind


def test_large_matrices():
    for shape in ((3, 512, 4608), (1, 2304, 2304)):
        G = gradient(*shape, "falling", seed=1)
        assert rel(run(G, B.F32), orthogonal(G)) <= TOL[B.F32]


@pytest.mark.parametrize("steps", [1, 2, 3, 8])
@pytest.mark.parametrize("shape", [(2, 64, 64), (2, 50, 300), (1, 300, 150)])
def test_steps(shape, steps):
    G = gradient(*shape, "gaussian", seed=steps)
    assert rel(run(G, B.F32, steps), orthogonal(G, steps)) <= TOL[B.F32]


def test_singular_values_come_near_one():
    G = gradient(1, 96, 400, "gaussian", seed=3)
    s = torch.linalg.svdvals(run(G, B.F32)[0].double())
    assert 0.6 < float(s.min()) and float(s.max()) < 1.25


@pytest.mark.parametrize("shape", [(3, 64, 64), (3, 64, 300), (3, 300, 64), (3, 100, 130)])
def test_scales_and_zeros(shape):
    """A matrix of zeros stays zeros; any other scale that float holds gives the same result, up to what 1e-7 beside a norm is."""
    G = gradient(*shape, "gaussian", seed=2)
    want = orthogonal(G)
    for scale in (1e-30, 1e-3, 1e10, 1e34):
        x = G * scale
        x[1] = 0
        o = run(x, B.F32)
        assert bool((o[1] == 0).all())
        exact = orthogonal(x)
        for k in (0, 2):
            assert rel(o[k], exact[k]) <= TOL[B.F32], scale
    assert rel(run(G * 1e10, B.F32), want) <= 2 * TOL[B.F32]


@pytest.mark.parametrize("shape", [(3, 64, 64), (3, 64, 300), (3, 130, 100)])
def test_non_finite_numbers_stay_in_their_matrix(shape):
    G = gradient(*shape, "gaussian", seed=2)
    for bad in (torch.nan, torch.inf, -torch.inf):
        x = G.clone()
        x[1, 3, 7] = bad
        o = run(x, B.F32)
        assert bool(torch.isnan(o[1]).any())
        want = orthogonal(G)
        for k in (0, 2):
            assert rel(o[k], want[k]) <= TOL[B.F32]


@pytest.mark.parametrize("shape", [(2, 64, 64), (2, 60, 500), (2, 500, 60), (1, 256, 130)])
def test_bfloat16_gradients_and_result_in_place(shape):
    G = gradient(*shape, "gaussian", seed=5).to(torch.bfloat16)
    want = orthogonal(G)
    assert rel(run(G, B.F32), want) <= TOL[B.F32]
    d = B.make_muon_desc(shape[1], shape[2], batch=shape[0], dtype=B.BF16, grad_dtype=B.BF16)
    call(d, B.MUON_ORTHOGONALISE, G, G)
    assert rel(G, want) <= TOL[B.BF16]


@pytest.mark.parametrize("nesterov", [0, 1])
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape", [(1, 64, 64), (4, 64, 576), (2, 257, 33), (2, 33, 257), (1, 1, 7), (3, 128, 200), (2, 1000, 129), (1, 65, 1001)])
def test_step(shape, dtype, nesterov):
    from gpu_util import Guarded
    g = torch.Generator(device=DEV)
    g.manual_seed(sum(shape))
    M, W = Guarded(shape, torch.float32), Guarded(shape, TYPES[dtype])
    M.t.copy_(torch.randn(shape, generator=g, device=DEV) * 1e-3)
    W.t.copy_(torch.randn(shape, generator=g, device=DEV))
    d = B.make_muon_desc(shape[1], shape[2], batch=shape[0], dtype=dtype, nesterov=nesterov)
    m, w = M.t.double(), W.t.double()
    for k in range(2):
        G = gradient(*shape, "gaussian", seed=k)
        m = 0.95 * m + G.double()
        u = G.double() + 0.95 * m if nesterov else m
        w = 0.99 * w - 0.5 * orthogonal(u)
        call(d, B.MUON_STEP, G, M.t, W.t, hyper=(0.95, 0.99, 0.5))
        assert rel(M.t, m) <= 1e-6
        assert rel(W.t, w) <= TOL[dtype]
        w = W.t.double()
    M.check("M")
    W.check("W")


def test_same_bits_again_and_on_another_stream():
    for shape in ((2, 64, 64), (2, 64, 1000), (2, 300, 500)):
        G = gradient(*shape, "falling", seed=4)
        first = run(G, B.F32).clone()
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            again = run(G, B.F32)
        torch.cuda.synchronize()
        assert torch.equal(first, again)


def test_captured_in_a_graph():
    for shape in ((2, 64, 500), (1, 200, 300)):
        G = gradient(*shape, "falling", seed=4)
        d = B.make_muon_desc(shape[1], shape[2], batch=shape[0], dtype=B.F32)
        want = run(G, B.F32).clone()
        O = torch.empty_like(G)
        ws = torch.empty(B.cac_muon_workspace_size(d, B.MUON_ORTHOGONALISE), dtype=torch.uint8, device=DEV)
        B.cac_orthogonalise(d, G, O, ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.cac_orthogonalise(d, G, O, ws)
        for _ in range(3):
            O.fill_(9)
            ws.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(O, want)
