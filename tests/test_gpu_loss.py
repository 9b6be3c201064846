"""Softmax cross entropy of a linear classifier on the GPU, against a plain implementation in 64 bits.

Tolerances.  float: a product keeps 22 bits or more and a sum of n terms loses at most sqrt(n) roundings of 2^-24 of
its largest partial sum in the mean; with logits of a spread of 2 over up to 2048 features that is below 2e-6 of a
logit's scale, so losses agree to 1e-5 and gradients (sums of such) to 2e-5 in the 2-norm.  bfloat16: inputs are
exact, losses are as for float; a gradient meets two roundings of 2^-9 at most (of the logits' gradients and of the
result), so 2^-8 in the 2-norm."""
import numpy as np
import pytest
import torch

from paper_2409_11902_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {B.F32: torch.float32, B.BF16: torch.bfloat16}
LOSS_TOL, GRAD_TOL = 1e-5, {B.F32: 2e-5, B.BF16: 2.0 ** -8}


def make(T, D, V, dtype, bias=1, out=0.0, seed=0, ld_h=0, ld_w=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    td = TYPES[dtype]

    def rows(n, ld, std):
        return (torch.randn(n, ld or D, generator=g, device=DEV) * std).to(td)

    t = {"H": rows(T, ld_h, 1.0), "W": rows(V, ld_w, 2.0 / D ** 0.5)}
    t["labels"] = torch.randint(0, V, (T,), generator=g, device=DEV)
    t["labels"][torch.rand(T, generator=g, device=DEV) < out] = -100
    t["gloss"] = torch.rand(T, generator=g, device=DEV) - 0.2
    t["b"] = (torch.randn(V, generator=g, device=DEV) * 0.5).to(td) if bias else None
    t["desc"] = B.make_loss_desc(T, D, V, dtype=dtype, has_bias=bias, ld_h=ld_h, ld_w=ld_w)
    return t


def reference(t, ignore=-100):
    """loss, lse, dH, dW, db in 64 bits; rows that do not count are not looked at."""
    d = t["desc"]
    T, D, V = d.T, d.D, d.V
    labels = t["labels"]
    live = ((labels >= 0) & (labels < V) & (labels != ignore)).nonzero().squeeze(1)
    h, w, y = t["H"][live, :D].double(), t["W"][:, :D].double(), labels[live]
    z = h @ w.t()
    if t["b"] is not None:
        z = z + t["b"].double()
    lse = torch.logsumexp(z, 1)
    at = torch.arange(len(live), device=DEV)
    r = {k: torch.zeros(T, dtype=torch.float64, device=DEV) for k in ("loss", "lse")}
    zy = z[at, y]
    r["lse"][live] = lse
    r["loss"][live] = torch.where(zy == -torch.inf, torch.inf, lse - zy)
    p = torch.where((lse == -torch.inf).unsqueeze(1), 0.0, (z - lse.unsqueeze(1)).exp())
    p[at, y] -= 1
    p = p * t["gloss"][live].double().unsqueeze(1)
    r["dH"] = torch.zeros(T, D, dtype=torch.float64, device=DEV)
    r["dH"][live] = p @ w
    r["dW"], r["db"] = p.t() @ h, p.sum(0)
    return r


def workspace(d, op):
    """Exactly what is asked for, with canaries behind it."""
    n = B.cac_loss_workspace_size(d, op)
    raw = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device=DEV)
    return raw, raw[:n]


def run(t, want=("dH", "dW", "db"), ws_fill=None):
    from gpu_util import Guarded
    d = t["desc"]
    td = t["H"].dtype
    out = {"loss": Guarded((d.T,), torch.float32), "lse": Guarded((d.T,), torch.float32), "dH": Guarded((d.T, d.D), td),
           "dW": Guarded((d.V, d.D), td), "db": Guarded((d.V,), td)}
    raw, ws = workspace(d, B.LOSS_FWD)
    B.cac_loss_fwd(d, t["H"], t["W"], t["b"], t["labels"], out["loss"].t, out["lse"].t, ws)
    raw2, ws2 = workspace(d, B.LOSS_BWD)
    B.cac_loss_bwd(d, t["H"], t["W"], t["b"], t["labels"], out["lse"].t, t["gloss"],
                   *(out[k].t if k in want else None for k in ("dH", "dW", "db")), ws2)
    torch.cuda.synchronize()
    for name, o in out.items():
        o.check(name)
    for r, w in ((raw, ws), (raw2, ws2)):
        assert bool((r[len(w):] == 0xA5).all()), "a write past the workspace"
    for k in ("dH", "dW", "db"):
        if k not in want:
            assert out[k].untouched_fraction() == 1.0
    return {k: o.t for k, o in out.items()}


def rel(a, b):
    n = b.norm()
    return float((a.double() - b).norm() / n) if n > 0 else float(a.double().norm())


def check(t, got, want=("dH", "dW", "db"), ignore=-100):
    r = reference(t, ignore)
    for k in ("loss", "lse"):
        fine = torch.isfinite(r[k])
        assert torch.equal(torch.isfinite(got[k]), fine), k
        assert torch.equal(got[k][~fine].double(), r[k][~fine]), k
        scale = 1 + r["lse"][torch.isfinite(r["lse"])].abs().max() if fine.any() else 1
        assert float((got[k].double() - r[k])[fine].abs().max() if fine.any() else 0) <= LOSS_TOL * float(scale), k
    for k in want:
        assert rel(got[k], r[k]) <= GRAD_TOL[t["desc"].dtype], (k, rel(got[k], r[k]))


SHAPES = [
    (1, 1, 1), (1, 8, 2), (1, 512, 1000), (2, 7, 5), (3, 64, 777), (17, 2048, 333), (63, 100, 64), (64, 64, 65), (65, 72, 129),
    (64, 2048, 1000), (129, 1024, 64), (200, 2047, 100), (256, 513, 5001), (300, 512, 21841), (1000, 33, 4099), (1031, 136, 20000),
]


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape", SHAPES)
def test_loss_and_gradients(shape, dtype):
    t = make(*shape, dtype, bias=sum(shape) % 2, out=0.3 if shape[0] > 2 else 0.0, seed=sum(shape))
    check(t, run(t))


@pytest.mark.parametrize("dtype,shape", [(B.BF16, (4096, 256, 40000)), (B.F32, (2048, 128, 50257)), (B.BF16, (20, 128, 600000)),
                                         (B.BF16, (4096, 256, 140000)), (B.F32, (2048, 128, 140000)), (B.F32, (20, 128, 600000))])
def test_classes_in_pieces(dtype, shape):
    t = make(*shape, dtype, out=0.1, seed=4)
    if shape[0] * shape[2] * (4 if dtype == B.F32 else 2) > 1 << 30 or shape[2] > 1 << 19:
        assert " 1 pieces" not in B.cac_loss_describe_plan(t["desc"], B.LOSS_BWD)
    check(t, run(t))


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("T", [1, 15, 17, 31, 33, 48, 64, 65, 100, 127, 128, 300])
@pytest.mark.parametrize("D,ld_h,ld_w", [(96, 0, 0), (98, 0, 0), (99, 0, 0), (96, 98, 100), (130, 131, 0), (128, 0, 129), (1, 0, 0), (2, 3, 4), (514, 516, 520)])
def test_few_rows_of_any_stride(T, D, ld_h, ld_w, dtype):
    t = make(T, D, 333, dtype, bias=D % 2, out=0.3 if T > 15 else 0.0, seed=T + D, ld_h=ld_h, ld_w=ld_w)
    check(t, run(t))


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("T", [5, 40, 64, 65, 500])
def test_rows_left_out_are_not_read(T, dtype):
    """NaN, infinities and the type's largest numbers in rows that do not count reach nothing."""
    t = make(T, 136, 300, dtype, out=0.5, seed=T)
    t["labels"][0], t["labels"][1], t["labels"][2] = -1, 300, -100
    t["labels"][3] = 7
    gone = (t["labels"] < 0) | (t["labels"] >= 300)
    t["H"][gone] = torch.nan
    t["H"][0], t["H"][1] = torch.inf, torch.finfo(t["H"].dtype).max
    t["gloss"][gone] = torch.nan
    got = run(t)
    check(t, got)
    assert bool((got["loss"][gone] == 0).all()) and bool((got["lse"][gone] == 0).all()) and bool((got["dH"][gone] == 0).all())


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("T", [3, 100])
def test_every_row_left_out(T, dtype):
    t = make(T, 64, 50, dtype)
    t["labels"][:] = -100
    t["H"][:] = torch.nan
    got = run(t)
    for k, v in got.items():
        assert bool((v == 0).all()), k


def test_ignore_index_that_is_a_class():
    t = make(90, 64, 20, B.F32, seed=2)
    t["desc"].ignore_index = 3
    t["labels"][::4] = 3
    check(t, run(t), ignore=3)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("T", [6, 80])
def test_masked_classes(T, dtype):
    """-inf in b takes a class out of every row's distribution; a row whose label is masked loses infinitely."""
    t = make(T, 64, 200, dtype, seed=9)
    t["labels"][:] = torch.arange(T, device=DEV) % 100
    t["b"][100:] = -torch.inf
    got = run(t)
    check(t, got)
    assert float(got["dW"][100:].double().abs().max()) == 0.0
    t["b"][:] = 0.0
    t["b"][2] = -torch.inf
    t["labels"][1] = 2
    got = run(t)
    check(t, got)
    assert float(got["loss"][1]) == np.inf
    t["b"][:] = -torch.inf
    check(t, run(t))
    t["b"][:] = torch.finfo(t["b"].dtype).min
    got = run(t)
    assert bool(torch.isfinite(got["loss"]).all()) or dtype == B.F32   # (the lowest number plus a logit is itself)
    assert all(bool(torch.isfinite(got[k]).all()) for k in ("dH", "dW", "db"))


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("ld", [(72, 80), (65, 67), (64, 67), (67, 64)])
def test_row_strides(ld, dtype):
    for T in (30, 150):
        t = make(T, 64, 130, dtype, ld_h=ld[0], ld_w=ld[1], seed=ld[0])
        if ld[0] > 64:
            t["H"][:, 64:] = torch.nan
        if ld[1] > 64:
            t["W"][:, 64:] = torch.nan
        check(t, run(t))


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("want", [("dH",), ("dW",), ("db",), ("dH", "db"), ("dW", "db")])
def test_gradients_not_asked_for(want, dtype):
    for shape in ((30, 64, 100), (300, 264, 9000)):
        t = make(*shape, dtype, seed=3)
        check(t, run(t, want), want)


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("scale", [1e-20, 1e-6, 1e15])
def test_scales_of_rows_gradients(scale, dtype):
    """Gradients of rows are of any size; equal ones lose nothing, zeros give zeros, an infinite one spoils its row of dH alone."""
    for T in (20, 90):
        t = make(T, 64, 50, dtype, seed=8)
        t["gloss"] *= scale
        check(t, run(t))
        t["gloss"][:] = 0
        got = run(t)
        assert all(bool((got[k] == 0).all()) for k in ("dH", "dW", "db"))
        t["gloss"][:] = scale
        t["gloss"][4] = torch.inf
        got = run(t)
        rest = torch.arange(T, device=DEV) != 4
        assert bool(torch.isfinite(got["dH"][rest]).all()) and not bool(torch.isfinite(got["dH"][4]).all())


def test_float_operands_of_uneven_scales():
    """Rows and weights over twelve orders of magnitude in one matrix: as far as the largest one's logits are concerned."""
    t = make(100, 128, 300, B.F32, seed=5)
    t["H"] *= 10.0 ** torch.linspace(-12, 0, 100, device=DEV).unsqueeze(1)
    t["W"] *= 10.0 ** torch.linspace(0, -12, 300, device=DEV).unsqueeze(1)
    check(t, run(t))
    for scale_h, scale_w in ((1e-18, 1e17), (1e25, 1e-25), (1e-30, 1.0)):
        t = make(100, 128, 300, B.F32, seed=5)
        t["H"] *= scale_h
        t["W"] *= scale_w
        got, want = run(t), reference(t)
        assert rel(got["lse"], want["lse"]) <= LOSS_TOL
        assert rel(got["dW"] / scale_h, want["dW"] / scale_h) <= GRAD_TOL[B.F32]
        assert rel(got["dH"] / scale_w, want["dH"] / scale_w) <= GRAD_TOL[B.F32]


def test_non_finite_numbers_stay_with_their_rows():
    for T in (40, 200):
        t = make(T, 64, 90, B.BF16, seed=6)
        t["H"][3, 5] = torch.nan
        got = run(t)
        rest = torch.arange(T, device=DEV) != 3
        assert bool(torch.isnan(got["loss"][3])) and bool(torch.isfinite(got["loss"][rest]).all())
        assert bool(torch.isnan(got["dH"][3]).all()) and bool(torch.isfinite(got["dH"][rest]).all())


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_gradient_against_differences(dtype):
    """The loss's own differences along directions of H, W and b, where the operands can be moved by exact amounts."""
    for T in (24, 120):
        t = make(T, 64, 150, dtype, seed=12)
        got = run(t)
        g = torch.Generator(device=DEV)
        g.manual_seed(1)
        eps = 2.0 ** -4
        for name, grad in (("H", "dH"), ("W", "dW"), ("b", "db")):
            base = (t[name].float() * 64).round() / 64                # a grid on which x + eps and x - eps are numbers of the type
            base = base.clamp(-2, 2)
            t2 = dict(t)
            t2[name] = base.to(t[name].dtype)
            got = run(t2)
            step = (torch.randint(0, 2, base.shape, generator=g, device=DEV) * 2 - 1).float() * eps / 64
            sums = []
            for sign in (1, -1):
                t3 = dict(t2)
                t3[name] = (base + sign * step)
                if dtype == B.BF16:                                    # (the step is kept exact by moving few elements at a time)
                    few = torch.rand(base.shape, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV) < 0.05
                    t3[name] = torch.where(few, base + sign * 2.0 ** -3 * step.sign(), base)
                moved = t3[name] - base
                t3[name] = t3[name].to(t[name].dtype)
                assert torch.equal(t3[name].float() - base, moved) or dtype == B.F32
                loss = torch.empty(T, device=DEV)
                raw, ws = workspace(t["desc"], B.LOSS_FWD)
                B.cac_loss_fwd(t["desc"], t3["H"], t3["W"], t3["b"], t3["labels"], loss, torch.empty_like(loss), ws)
                sums.append((float((loss.double() * t["gloss"].double()).sum()), moved.double()))
            slope = float((got[grad].double() * (sums[0][1] - sums[1][1])).sum())
            size = float(got[grad].double().norm() * (sums[0][1] - sums[1][1]).norm())
            # differences: rounding of the losses, third derivatives, and a gradient's own rounding
            assert abs((sums[0][0] - sums[1][0]) - slope) <= 1e-2 * size + 1e-5 * T, (name, T)


def test_same_bits_again_and_on_another_stream():
    for shape, dtype in (((50, 64, 300), B.BF16), ((700, 264, 3000), B.F32), ((600, 264, 20000), B.BF16)):
        t = make(*shape, dtype, out=0.2, seed=1)
        first = {k: v.clone() for k, v in run(t).items()}
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            again = run(t)
        torch.cuda.synchronize()
        for k in first:
            assert torch.equal(first[k], again[k]), k


def test_captured_in_a_graph():
    t = make(100, 128, 500, B.BF16, out=0.1, seed=3)
    d = t["desc"]
    want = {k: v.clone() for k, v in run(t).items()}
    out = {k: torch.empty_like(v) for k, v in want.items()}
    ws = torch.empty(max(B.cac_loss_workspace_size(d, op) for op in (0, 1)), dtype=torch.uint8, device=DEV)

    def step():
        B.cac_loss_fwd(d, t["H"], t["W"], t["b"], t["labels"], out["loss"], out["lse"], ws)
        B.cac_loss_bwd(d, t["H"], t["W"], t["b"], t["labels"], out["lse"], t["gloss"], out["dH"], out["dW"], out["db"], ws)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for v in out.values():
            v.fill_(7)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(out[k], want[k]), k
