"""The dense layer with its ending on the GPU, against its formulas in 64 bits.

Tolerances.  A product's sum of D terms rounds partial sums of at most a = sum |x| |w| (+ |b|) to 2^-23 (the matrix instructions may
truncate): roundings of independent signs add up to sqrt(D) of them in the mean, four times that and eight more are allowed,
u = 2^-23 (4 sqrt(D) + 8) a.  The derivatives of the activations are at most 1.13 and their derivatives below 0.8 (GELU), 0.5 (SILU); evaluating them
costs 2^-20 of |u| (of 1 for the derivative).  Results are rounded to half a step.  bfloat16 rounds dU to half a step of itself before it is multiplied.
ReLU's derivative jumps, so its inputs are small whole numbers, whose products are exact.  In the 2-norm a float result is within
1e-5 and a bfloat16 one within 2^-8: its two roundings of at most 2^-8 an element are of a spread below 2^-9 each.  That is so of
many; where dU has fewer than 64 elements they may all err to one side, and the bound is (1 + 2^-8)^2 - 1."""
import numpy as np
import pytest
import torch

from block_util import DEV, HALF, TYPES, Scratch, act, close, keep_factor, make_rng, rel, rows
from paper_2409_11902_amd import binding as B

pytestmark = pytest.mark.gpu
NORM2 = {B.F32: 1e-5, B.BF16: 2.0 ** -8}
SITE = 11


def make(T, D, N, dtype, kind=B.ACT_NONE, bias=1, res=0, p=0.0, alpha=1.0, ld_x=0, ld_w=0, ld_r=0, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + T + 3 * D + 5 * N)
    whole = kind == B.ACT_RELU

    def matrix(n, cols, ld, std):
        t = rows(g, n, cols, ld, dtype, 1.5 if whole else std)
        if whole:
            t.copy_(t.float().round().clamp(-3, 3))
        return t

    t = {"X": matrix(T, D, ld_x, 1.0), "W": matrix(N, D, ld_w, D ** -0.5), "dY": rows(g, T, N, 0, dtype)}
    t["b"] = (torch.randn(N, generator=g, device=DEV) * 2).round().div(2).to(TYPES[dtype]) if bias else None
    t["R"] = rows(g, T, N, ld_r, dtype, 2.0) if res else None
    t["rng"] = make_rng(17 + seed, 5)
    t["desc"] = B.make_linear_desc(T, D, N, dtype=dtype, has_bias=bias, act=kind, alpha=alpha, p=p, site=SITE, ld_x=ld_x, ld_w=ld_w, ld_r=ld_r)
    return t


def reference(t):
    """Values and the bounds of their errors."""
    d = t["desc"]
    half, x, w = HALF[d.dtype], t["X"].double(), t["W"].double()
    eps = 2.0 ** -23

    def slack(terms):
        return eps * (4 * terms ** 0.5 + 8)

    b = t["b"].double() if t["b"] is not None else 0.0
    u = x @ w.t() + b
    du = slack(d.D) * (x.abs() @ w.abs().t() + (b.abs() if t["b"] is not None else 0.0))
    y, s = act(d.act, u)
    ds = (0.8 * du + 2.0 ** -20) if d.act in (B.ACT_GELU, B.ACT_SILU) else torch.zeros_like(u)
    keep = keep_factor(d.T, d.N, d.drop_p, d.site, t["rng"].tolist()).to(DEV)
    alpha = float(np.float32(d.alpha))
    f = abs(alpha) * float(keep.max()) if bool(keep.any()) else 0.0
    r = {"Y": torch.where(keep > 0, alpha * keep * y, 0.0) + (t["R"].double() if t["R"] is not None else 0.0)}
    e = {"Y": abs(alpha) * keep * (1.13 * du + (2.0 ** -20 * u.abs() if d.act else 0.0)) + 4 * eps * (r["Y"].abs() + alpha * keep * y.abs()).abs() + half * r["Y"].abs()}
    dy = t["dY"].double()
    g = torch.where(keep > 0, dy * s, 0.0)            # without the factor
    eg = torch.where(keep > 0, dy.abs() * ds, 0.0)
    eb = f * (eg.sum(0) + slack(d.T) * g.abs().sum(0))
    if d.act != B.ACT_NONE:
        eg = eg + half * g.abs() + 2 * eps * g.abs()
    sign = 1.0 if alpha >= 0 else -1.0
    r["dX"], r["dW"], r["db"] = sign * f * (g @ w), sign * f * (g.t() @ x), sign * f * g.sum(0)
    e["dX"] = f * (eg @ w.abs() + slack(d.N) * (g.abs() @ w.abs())) + half * r["dX"].abs()
    e["dW"] = f * (eg.t() @ x.abs() + slack(d.T) * (g.abs().t() @ x.abs())) + half * r["dW"].abs()
    e["db"] = eb + half * r["db"].abs()
    return r, e


def forward(t):
    from gpu_util import Guarded
    d = t["desc"]
    out, s = Guarded((d.T, d.N), TYPES[d.dtype]), Scratch(B.cac_linear_workspace_size(d, B.LINEAR_FWD))
    B.cac_linear_fwd(d, t["X"], t["W"], t["b"], t["R"], t["rng"], out.t, s.ws)
    torch.cuda.synchronize()
    out.check("Y")
    s.check()
    return out.t


def backward(t, want=("dX", "dW", "db")):
    from gpu_util import Guarded
    d, td = t["desc"], TYPES[t["desc"].dtype]
    o = {"dX": Guarded((d.T, d.D), td), "dW": Guarded((d.N, d.D), td), "db": Guarded((d.N,), td)}
    s = Scratch(B.cac_linear_workspace_size(d, B.LINEAR_BWD))
    B.cac_linear_bwd(d, t["X"], t["W"], t["b"], t["dY"], t["rng"], *(o[k].t if k in want else None for k in ("dX", "dW", "db")), s.ws)
    torch.cuda.synchronize()
    s.check()
    for k, v in o.items():
        v.check(k)
        if k not in want:
            assert bool((v.raw == 0xA5).all())
    return {k: o[k].t for k in want}


def check(t, fwd=True, bwd=True):
    r, e = reference(t)
    got = {"Y": forward(t)} if fwd else {}
    if bwd:
        got.update(backward(t))
    for k, v in got.items():
        close(k, v, r[k], e[k])
        few = t["desc"].dtype == B.BF16 and t["desc"].T * t["desc"].N < 64
        assert rel(v, r[k]) <= ((1 + 2.0 ** -8) ** 2 - 1 if few else NORM2[t["desc"].dtype]), (k, rel(v, r[k]))


SHAPES = [
    (1, 1, 1), (1, 8, 8), (1, 512, 2048), (2, 7, 5), (3, 64, 77), (17, 2048, 333), (31, 100, 64), (32, 64, 32), (33, 72, 31), (64, 2048, 1000),
    (65, 72, 129), (129, 1024, 64), (200, 2047, 100), (256, 513, 1001), (300, 512, 2560), (1000, 33, 515), (1031, 136, 1000), (2049, 264, 8), (4100, 24, 40),
]


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape", SHAPES)
def test_plain(shape, dtype):
    check(make(*shape, dtype, bias=sum(shape) % 2, res=shape[0] % 2))


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("kind", [B.ACT_RELU, B.ACT_GELU, B.ACT_SILU])
@pytest.mark.parametrize("shape", [(1, 1, 1), (1, 512, 2048), (5, 64, 77), (31, 96, 65), (64, 2048, 1000), (200, 2047, 100), (300, 512, 640), (1031, 136, 1000)])
def test_activations_with_dropout(shape, kind, dtype):
    check(make(*shape, dtype, kind, bias=(sum(shape) + kind) % 2, res=kind % 2, p=0.2 if shape[0] > 1 else 0.0, alpha=0.5))


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("p", [0.1, 0.5, 1.0])
@pytest.mark.parametrize("shape", [(1, 64, 9), (16, 2048, 515), (257, 96, 64), (700, 200, 1003)])
def test_dropout_without_activation(shape, p, dtype):
    check(make(*shape, dtype, bias=1, res=1, p=p, alpha=-1.5))


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("T", [1, 4, 16, 31, 33, 64, 100, 300])
@pytest.mark.parametrize("D,ld_x,ld_w", [(96, 0, 0), (98, 0, 0), (99, 0, 0), (96, 98, 100), (130, 131, 0), (128, 0, 129), (96, 104, 112), (1, 0, 0), (2, 3, 4)])
def test_rows_of_any_stride(T, D, ld_x, ld_w, dtype):
    check(make(T, D, 203, dtype, B.ACT_SILU if D % 2 else B.ACT_NONE, res=1, ld_x=ld_x, ld_w=ld_w, ld_r=205 + D % 4))


@pytest.mark.parametrize("dtype,shape", [(B.BF16, (2048, 1024, 4096)), (B.BF16, (4096, 512, 2056)), (B.F32, (1536, 1024, 2048)), (B.BF16, (16, 8192, 2048)),
                                         (B.BF16, (1000, 1000, 1000)), (B.F32, (16, 8192, 512))])
def test_large(shape, dtype):
    check(make(*shape, dtype, B.ACT_GELU, res=1, p=0.1))


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("kind", [B.ACT_NONE, B.ACT_GELU])
@pytest.mark.parametrize("want", [("dX",), ("dW",), ("db",), ("dX", "db"), ("dW", "db")])
def test_some_gradients(want, kind, dtype):
    t = make(70, 99, 131, dtype, kind, p=0.3)
    every = backward(t)
    some = backward(t, want)
    assert all(torch.equal(some[k], every[k]) for k in want)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape", [(3, 64, 40), (16, 4096, 520), (300, 64, 520), (300, 64, 519)])
def test_in_place_of_the_residual(shape, dtype):
    t = make(*shape, dtype, B.ACT_GELU, res=1, p=0.2)
    want = forward(t).clone()
    d = t["desc"]
    ws = torch.empty(B.cac_linear_workspace_size(d, B.LINEAR_FWD), dtype=torch.uint8, device=DEV)
    B.cac_linear_fwd(d, t["X"], t["W"], t["b"], t["R"], t["rng"], t["R"], ws)
    assert torch.equal(t["R"], want)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("T", [3, 40, 200])
def test_infinities_and_nan_stay_in_their_rows(T, dtype):
    t = make(T, 72, 100, dtype, B.ACT_NONE, res=1)
    clean, grads = forward(t).clone(), {k: v.clone() for k, v in backward(t).items()}
    t["X"][0, 3], t["R"][1, 5], t["dY"][2, 7] = float("nan"), float("inf"), float("inf")
    y = forward(t)
    assert bool(torch.isnan(y[0]).all()) and bool(torch.isinf(y[1, 5]))
    same = torch.ones_like(y, dtype=torch.bool)
    same[0], same[1, 5] = False, False
    assert torch.equal(y[same], clean[same])
    g = backward(t)
    assert not bool(torch.isfinite(g["dX"][2]).any()) and torch.equal(g["dX"][:2], grads["dX"][:2]) and torch.equal(g["dX"][3:], grads["dX"][3:])
    others = torch.arange(100, device=DEV) != 7
    columns = torch.arange(72, device=DEV) != 3
    assert torch.equal(g["dW"][others][:, columns], grads["dW"][others][:, columns]) and bool(torch.isnan(g["dW"][others][:, 3]).all())
    assert not bool(torch.isfinite(g["db"][7])) and torch.equal(g["db"][others], grads["db"][others])


@pytest.mark.parametrize("kind", [B.ACT_RELU, B.ACT_GELU, B.ACT_SILU])
def test_activations_at_their_ends(kind):
    """u from the bias alone: zeros, tiny numbers, the tails and beyond."""
    v = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e-3, -1e-3, 0.5, -0.5, 3.0, -3.0, -5.0, -8.0, -12.0, 12.0, 40.0, -40.0, 90.0, -90.0, 1e4, -1e4, 3e38], device=DEV)
    n = len(v)
    d = B.make_linear_desc(2, 8, n, dtype=B.F32, has_bias=1, act=kind)
    X, W, y = torch.zeros(2, 8, device=DEV), torch.zeros(n, 8, device=DEV), torch.empty(2, n, device=DEV)
    ws = torch.empty(max(16, B.cac_linear_workspace_size(d, B.LINEAR_BWD)), dtype=torch.uint8, device=DEV)
    B.cac_linear_fwd(d, X, W, v, None, None, y, ws)
    want, slope = act(kind, v.double())
    # u^2 / 2 is rounded before its exponential is taken: 2^-24 u^2 of the tail, beside 2^-20
    close("y", y[0], want, want.abs() * (2.0 ** -20 + 2.0 ** -22 * torch.minimum(v.double().abs(), torch.tensor(200.0, device=DEV)) ** 2) + 1e-37)
    db = torch.empty(n, device=DEV)
    B.cac_linear_bwd(d, X, W, v, torch.full((2, n), 0.5, device=DEV), None, None, None, db, ws)
    close("slope", db, slope, 2.0 ** -20 * (1 + slope.abs()))


@pytest.mark.parametrize("kind", [B.ACT_NONE, B.ACT_GELU, B.ACT_SILU])
def test_gradients_against_differences(kind):
    """Central differences of the formula in 64 bits along random directions: errors of h^2 = 1e-8 of third derivatives."""
    t = make(37, 50, 41, B.F32, kind, p=0.25, alpha=0.7)
    got = backward(t)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    keep = keep_factor(37, 41, 0.25, SITE, t["rng"].tolist()).to(DEV) * float(np.float32(0.7))

    def value(X, W, b):
        return float((keep * act(kind, X @ W.t() + b)[0] * t["dY"].double()).sum())

    at = [t[k].double() for k in ("X", "W", "b")]
    for i, name in enumerate(("dX", "dW", "db")):
        v = torch.randn(at[i].shape, generator=g, device=DEV, dtype=torch.float64)
        h = 1e-4
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * v, at[i] - h * v
        slope = (value(*up) - value(*down)) / (2 * h)
        size = float(got[name].double().norm() * v.norm())
        assert abs(float((got[name].double() * v).sum()) - slope) <= 2e-5 * size, name


@pytest.mark.parametrize("shape,kind", [((16, 4096, 512), B.ACT_GELU), ((300, 513, 515), B.ACT_SILU), ((512, 256, 512), B.ACT_NONE)])
def test_replays(shape, kind):
    """Captured together, replayed with eager work between, another step each time."""
    t = make(*shape, B.BF16, kind, res=1, p=0.1)
    d, td = t["desc"], torch.bfloat16
    ws = torch.empty(max(B.cac_linear_workspace_size(d, op) for op in (B.LINEAR_FWD, B.LINEAR_BWD)), dtype=torch.uint8, device=DEV)
    o = [torch.empty(s, dtype=td, device=DEV) for s in ((d.T, d.N), (d.T, d.D), (d.N, d.D), (d.N,))]

    def both(o):
        B.cac_linear_fwd(d, t["X"], t["W"], t["b"], t["R"], t["rng"], o[0], ws)
        B.cac_linear_bwd(d, t["X"], t["W"], t["b"], t["dY"], t["rng"], *o[1:], ws)

    both(o)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(o)
    for step in range(3):
        t["rng"][1] = step
        graph.replay()
        got = [x.clone() for x in o]
        want = [torch.empty_like(x) for x in o]
        ws.fill_(0xFF)
        both(want)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_streams_with_workspaces_of_their_own():
    ts = [make(260, 512, 640, B.BF16, B.ACT_GELU, p=0.1, seed=s) for s in range(2)]
    want = [forward(t).clone() for t in ts]
    streams = [torch.cuda.Stream() for _ in ts]
    out = [torch.empty_like(w) for w in want]
    ws = [torch.empty(max(16, B.cac_linear_workspace_size(t["desc"], B.LINEAR_FWD)), dtype=torch.uint8, device=DEV) for t in ts]
    torch.cuda.synchronize()
    for _ in range(5):
        for t, s, o, w in zip(ts, streams, out, ws):
            B.cac_linear_fwd(t["desc"], t["X"], t["W"], t["b"], t["R"], t["rng"], o, w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
