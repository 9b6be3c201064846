"""A tensor that a call of the residual block cannot do without and that is None: the binding passes it on, and the library says which one is missing,
as it does of the other calls.  No GPU is needed: each call is refused before anything is launched."""
from types import SimpleNamespace

import pytest
import torch

from paper_2409_11902_amd import binding as B

T, D, N = 8, 16, 24
STREAM = SimpleNamespace(cuda_stream=None)


def buffer():
    raw = torch.empty(4096 + 16, dtype=torch.uint8)
    return raw[-raw.data_ptr() % 16:]


def dropout(**t):
    B.cac_dropout(B.make_dropout_desc(T, D, p=0.5), t["X"], None, t["rng"], t["Y"], stream=STREAM)


def linear_fwd(**t):
    B.cac_linear_fwd(B.make_linear_desc(T, D, N, has_bias=1, p=0.5), t["X"], t["W"], t["b"], None, t["rng"], t["Y"], stream=STREAM)


def linear_bwd(**t):
    B.cac_linear_bwd(B.make_linear_desc(T, D, N, has_bias=1, act=B.ACT_GELU, p=0.5), t["X"], t["W"], t["b"], t["dY"], t["rng"], buffer(), None, None,
                     stream=STREAM)


def norm_fwd(**t):
    B.cac_block_norm_fwd(B.make_block_norm_desc(T, D, post=1, pre=1, gate_rows=T, p=0.5), t["F"], None, t["gate"], None, None, None, None, t["rng"], buffer(),
                         t["H"], stream=STREAM)


def norm_bwd(**t):
    B.cac_block_norm_bwd(B.make_block_norm_desc(T, D, post=1, pre=1, gate_rows=T, p=0.5), t["F"], t["S"], t["gate"], None, None, None, t["dH"], None,
                         t["rng"], buffer(), None, None, None, None, None, None, stream=STREAM)


@pytest.mark.parametrize("call,names", [(dropout, ("X", "rng", "Y")), (linear_fwd, ("X", "W", "b", "rng", "Y")), (linear_bwd, ("X", "W", "b", "dY", "rng")),
                                        (norm_fwd, ("F", "gate", "rng", "H")), (norm_bwd, ("F", "S", "gate", "dH", "rng"))])
def test_a_missing_tensor_is_named(call, names):
    for missing in names:
        with pytest.raises(B.CacError, match=rf"\b{missing} is NULL") as e:
            call(**{n: None if n == missing else buffer() for n in names})
        assert e.value.args and "error -1" in str(e.value)
