"""Dense layers whose products take tiles of 256 x 256, in either pass, at rows, columns and terms that are no multiples of a tile's: against the formulas
in 64 bits, with the tolerances of the dense layer's other tests."""
import re

import pytest
import torch

from test_gpu_linear import backward, check, forward, make

from paper_2409_11902_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def tiles(d, op):
    """{product: (tile, slices)} of those that a call has."""
    return {m[1]: (m[2], int(m[3])) for m in re.finditer(r"(pre-activation|dX|dW): tile ([\dx ]+) in (\d+) slices", B.cac_linear_describe_plan(d, op))}


# the products that take 256 x 256, and whether their sums are formed in slices
CASES = [
    ((4097, 2056, 4104), B.ACT_GELU, {"dX": False, "dW": False}),
    ((2049, 8200, 2056), B.ACT_SILU, {"dX": False, "dW": False}),
    ((4001, 4008, 4000), B.ACT_GELU, {"Y": False, "u": False, "dX": False, "dW": False}),
    ((4001, 4008, 4000), B.ACT_NONE, {"Y": False, "dX": False, "dW": False}),
    ((3001, 4104, 4101), B.ACT_RELU, {"Y": False, "dX": False, "dW": False}),
    ((3001, 4099, 4104), B.ACT_SILU, {"Y": False, "dX": False, "dW": False}),
    ((659, 128, 20485), B.ACT_NONE, {"Y": False}),
    ((133, 8119, 17145), B.ACT_GELU, {"Y": True, "u": True}),
    ((4585, 9390, 134), B.ACT_GELU, {"dW": True}),
    ((22332, 1056, 147), B.ACT_GELU, {"dW": True}),
    ((137, 2358, 10074), B.ACT_GELU, {"dX": True}),
]


@pytest.mark.parametrize("shape,kind,large", CASES)
def test_large_tiles(shape, kind, large):
    t = make(*shape, B.BF16, kind, res=1, p=0.1, alpha=-0.5)
    fwd, bwd = tiles(t["desc"], B.LINEAR_FWD), tiles(t["desc"], B.LINEAR_BWD)
    for name, sliced in large.items():
        tile, slices = fwd["pre-activation"] if name == "Y" else bwd["pre-activation" if name == "u" else name]
        assert tile == "256" and (slices > 1) == sliced, (name, tile, slices)
    check(t)


@pytest.mark.parametrize("shape,kind", [((4097, 2056, 4104), B.ACT_GELU), ((4001, 4008, 4000), B.ACT_NONE), ((22332, 1056, 147), B.ACT_GELU), ((137, 2358, 10074), B.ACT_GELU)])
def test_again_and_each_gradient_alone(shape, kind):
    """The same bits a second time, and of a gradient that is asked for by itself."""
    t = make(*shape, B.BF16, kind, p=0.1)
    y, every = forward(t).clone(), {k: v.clone() for k, v in backward(t).items()}
    assert torch.equal(forward(t), y)
    again = backward(t)
    assert all(torch.equal(again[k], every[k]) for k in every)
    for k in every:
        assert torch.equal(backward(t, (k,))[k], every[k]), k
