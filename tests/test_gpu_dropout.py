"""Dropout on the GPU against its definition in 64 bits.

A result meets the rounding of the factor, of its product and of the sum with R (2^-24 each of |R| + |x|'s part, 4 of them at most) and,
bfloat16, one of 2^-8 of itself."""
import numpy as np
import pytest
import torch

from block_util import DEV, HALF, TYPES, close, keep_factor, limit_of, make_rng, philox, rows
from paper_2409_11902_amd import binding as B


def test_generator_gives_the_published_numbers():
    """The answers for counter and key of zeros and of all ones that the generator's authors publish."""
    assert [int(x) for x in philox((0, 0, 0, 0), (0, 0))] == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    f = 0xFFFFFFFF
    assert [int(x) for x in philox((f, f, f, f), (f, f))] == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def run(T, D, dtype, p, alpha=1.0, res=True, site=5, ld_x=0, ld_r=0, seed=0, rng=None, X=None, into=None):
    from gpu_util import Guarded
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + T + D)
    X = rows(g, T, D, ld_x, dtype) if X is None else X
    R = rows(g, T, D, ld_r, dtype, 2.0) if res else None
    rng = make_rng(seed * 7919 + 1, (seed << 33) + 3) if rng is None else rng
    out = Guarded((T, D), TYPES[dtype])
    d = B.make_dropout_desc(T, D, dtype=dtype, p=p, alpha=alpha, site=site, ld_x=ld_x, ld_r=ld_r)
    B.cac_dropout(d, X, R, rng, out.t)
    torch.cuda.synchronize()
    out.check()
    k = keep_factor(T, D, p, site, rng.tolist()).to(DEV)
    part = torch.where(k > 0, X.double() * k * float(np.float32(alpha)), 0.0)
    want = part + (R.double() if res else 0.0)
    size = part.abs() + (R.double().abs() if res else 0.0)
    close("Y", out.t, want, 4 * 2.0 ** -24 * size + HALF[dtype] * want.abs() * (dtype == B.BF16))
    return out.t, X, k


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("shape", [(1, 1), (1, 8), (1, 9), (3, 7), (7, 64), (64, 512), (33, 1001), (129, 130), (2, 40000), (70000, 3), (1031, 520)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5])
def test_dropout(shape, dtype, p):
    run(*shape, dtype, p, alpha=-0.75 if shape[1] % 2 else 1.0, res=shape[0] % 2 == 1, seed=shape[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("ld_x,ld_r", [(104, 0), (0, 112), (97, 98), (99, 0), (100, 100)])
@pytest.mark.parametrize("D", [96, 97, 1])
def test_strides(D, ld_x, ld_r, dtype):
    run(37, D, dtype, 0.25, ld_x=ld_x and max(ld_x, D), ld_r=ld_r and max(ld_r, D))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("p", [1e-5, 0.99999])
def test_one_in_65536(p, dtype):
    """The least and the most that 16 bits can tell from none and all."""
    assert limit_of(p) in (1, 65535)
    _, _, k = run(1000, 1003, dtype, p, seed=8)
    assert 0 < int((k == 0).sum()) < k.numel()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_everything_and_nothing(dtype):
    """p = 1 drops all; p below 2^-17 rounds to none, and rng is not asked for."""
    y, _, _ = run(9, 33, dtype, 1.0, res=False)
    assert not bool(y.any())
    x = torch.randn(9, 33, device=DEV).to(TYPES[dtype])
    y = torch.empty_like(x)
    B.cac_dropout(B.make_dropout_desc(9, 33, dtype=dtype, p=2.0 ** -18), x, None, None, y)
    assert torch.equal(x, y)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_what_is_dropped_is_zero_whatever_it_is(dtype):
    X = torch.full((50, 41), float("nan"), device=DEV).to(TYPES[dtype])
    X[:, ::2] = float("inf")
    d = B.make_dropout_desc(50, 41, dtype=dtype, p=0.5, site=5)
    y = torch.empty_like(X)
    rng = make_rng(3, 1)
    B.cac_dropout(d, X, None, rng, y)
    k = keep_factor(50, 41, 0.5, 5, rng.tolist()).to(DEV) > 0
    assert not bool(y[~k].any()) and bool((~torch.isfinite(y[k])).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("D", [64, 65])
def test_in_place_and_gradient(D, dtype):
    """Y over X and over R; the gradient is the call itself, <drop(x), y> = <x, drop(y)>."""
    y, X, k = run(40, D, dtype, 0.3, res=False, seed=2)
    rng = make_rng(2 * 7919 + 1, (2 << 33) + 3)
    d = B.make_dropout_desc(40, D, dtype=dtype, p=0.3, site=5)
    over = X.clone()
    B.cac_dropout(d, over, None, rng, over)
    assert torch.equal(over, y)
    R = torch.randn(40, D, device=DEV).to(TYPES[dtype])
    want = torch.empty_like(R)
    B.cac_dropout(d, X, R, rng, want)
    B.cac_dropout(d, X, R, rng, R)
    assert torch.equal(R, want)
    g = torch.randn(40, D, device=DEV).to(TYPES[dtype])
    gx = torch.empty_like(g)
    B.cac_dropout(d, g, None, rng, gx)
    assert torch.equal(gx == 0, (k == 0) | (g == 0))


@pytest.mark.gpu
def test_masks_of_steps_sites_and_keys_differ_and_keep_what_they_should():
    x = torch.ones(512, 1000, device=DEV)
    masks = []
    for seed, step, site in ((1, 0, 0), (1, 1, 0), (1, 0, 1), (2, 0, 0), (1, 1 << 32, 0), (1 << 32, 0, 0)):
        y = torch.empty_like(x)
        B.cac_dropout(B.make_dropout_desc(512, 1000, dtype=B.F32, p=0.2, site=site), x, None, make_rng(seed, step), y)
        masks.append(y != 0)
        # 512000 draws of probability 0.8: five times the spread is 5 sqrt(0.16 / 512000) = 0.0028
        assert abs(float(masks[-1].double().mean()) - 0.8) < 0.0028
    for i in range(len(masks)):
        for k in range(i):  # two independent masks agree in 0.68 of places, of spread 0.00065
            assert abs(float((masks[i] == masks[k]).double().mean()) - 0.68) < 0.0033


@pytest.mark.gpu
def test_replays_follow_the_step():
    """A captured call reads rng when it runs."""
    x, r = torch.randn(300, 200, device=DEV).bfloat16(), torch.randn(300, 200, device=DEV).bfloat16()
    d, rng, y = B.make_dropout_desc(300, 200, p=0.4), make_rng(9, 0), torch.empty_like(x)
    B.cac_dropout(d, x, r, rng, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cac_dropout(d, x, r, rng, y)
    seen = []
    for step in range(4):
        rng[1] = step
        graph.replay()
        got = y.clone()
        want = torch.empty_like(x)
        B.cac_dropout(d, x, r, rng, want)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        seen.append(got)
    assert all(not torch.equal(seen[0], s) for s in seen[1:])


@pytest.mark.gpu
def test_on_another_stream():
    x = torch.randn(1000, 1000, device=DEV)
    d, rng, want, y = B.make_dropout_desc(1000, 1000, dtype=B.F32, p=0.4), make_rng(9, 0), torch.empty_like(x), torch.empty_like(x)
    B.cac_dropout(d, x, None, rng, want)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    B.cac_dropout(d, x, None, rng, y, stream=s)
    s.synchronize()
    assert torch.equal(y, want)
