"""Orthogonalised updates whose outputs lie where something else of the call lies: refused before any launch, but for O over a G of its type."""
import pytest

from paper_2409_11902_amd import binding as B

MB = 1 << 20


# one launch a matrix, one a step, and products
@pytest.mark.parametrize("rows,cols", [(64, 64), (64, 1000), (300, 200)])
@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("grad_dtype", [B.F32, B.BF16])
def test_outputs_share_no_memory(rows, cols, dtype, grad_dtype):
    """These calls would touch the GPU if the check let them through."""
    L, d = B.lib(), B.make_muon_desc(rows, cols, batch=2, dtype=dtype, grad_dtype=grad_dtype)
    n = 2 * rows * cols
    of = {B.F32: 4, B.BF16: 2}
    sizes = {"G": n * of[grad_dtype], "M": n * 4, "W": n * of[dtype], "O": n * of[dtype], "ws": max(16, B.cac_muon_workspace_size(d, B.MUON_STEP))}
    at = {name: (k + 1) * 64 * MB for k, name in enumerate(sizes)}
    step = lambda p: L.cac_muon_step(d, p["G"], p["M"], p["W"], 0.9, 1.0, 0.1, p["ws"], sizes["ws"], None)
    orth = lambda p: L.cac_orthogonalise(d, p["G"], p["O"], p["ws"], sizes["ws"], None)
    used = B.cac_muon_workspace_size(d, B.MUON_STEP) > 0
    for call, pairs in ((step, (("M", "G"), ("W", "G"), ("M", "W"), ("M", "ws"), ("W", "ws"))), (orth, (("O", "G"), ("O", "ws")))):
        for out, other in pairs:
            if other == "ws" and not used:
                continue
            for place in (at[other] + (sizes[other] - 1) // 16 * 16, at[other] - (sizes[out] - 1) // 16 * 16):
                assert call({**at, out: place}) == B.ERR_INVALID_ARG, (out, other)
                assert out in L.cac_last_error().decode() and "shares memory" in L.cac_last_error().decode()
            if not (out == "O" and other == "G" and dtype == grad_dtype) and other != "ws":
                assert call({**at, out: at[other]}) == B.ERR_INVALID_ARG, (out, other)
