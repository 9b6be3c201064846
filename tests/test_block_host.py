"""What the residual block's entry points refuse, before anything is launched, and what they say about their plans.  No GPU is needed: a call that
were let through would fail at its launch with another code."""
import ctypes

import pytest

from paper_2409_11902_amd import binding as B

MB = 1 << 20
ALL = (B.F32, B.BF16)


def addresses(names):
    return {n: (k + 1) * 64 * MB for k, n in enumerate(names)}


class Linear:
    fwd = ("X", "W", "b", "R", "rng", "Y")
    bwd = ("X", "W", "b", "dY", "rng", "dX", "dW", "db")

    @staticmethod
    def call(d, op, ws=1 << 33, ws_bytes=None, **over):
        L = B.lib()
        names = Linear.fwd if op == B.LINEAR_FWD else Linear.bwd
        p = {**addresses(names), **over}
        if ws_bytes is None:
            n = ctypes.c_size_t()
            ws_bytes = n.value if L.cac_linear_workspace_size(d, op, ctypes.byref(n)) else n.value
        fn = L.cac_linear_fwd if op == B.LINEAR_FWD else L.cac_linear_bwd
        return fn(d, *(p[n] for n in names), ws, ws_bytes, None)


class Norm:
    fwd = ("F", "R", "gate", "w_post", "b_post", "w_pre", "b_pre", "rng", "S", "H")
    bwd = ("F", "S", "gate", "w_post", "b_post", "w_pre", "dH", "dS", "rng", "dR", "dF", "dgate", "dw_post", "db_post", "dw_pre", "db_pre")

    @staticmethod
    def call(d, op, ws=1 << 33, ws_bytes=None, **over):
        L = B.lib()
        names = Norm.fwd if op == B.BLOCK_NORM_FWD else Norm.bwd
        p = {**addresses(names), **over}
        if op == B.BLOCK_NORM_FWD:
            return L.cac_block_norm_fwd(d, *(p[n] for n in names), None)
        if ws_bytes is None:
            n = ctypes.c_size_t()
            L.cac_block_norm_workspace_size(d, op, ctypes.byref(n))
            ws_bytes = n.value
        return L.cac_block_norm_bwd(d, *(p[n] for n in names), ws, ws_bytes, None)


def refused(rc, code, word=""):
    assert rc == code, (rc, B.lib().cac_last_error())
    assert word in B.lib().cac_last_error().decode(), B.lib().cac_last_error()


def linear(**over):
    return B.make_linear_desc(**{**dict(T=40, D=64, N=48, has_bias=1, act=B.ACT_GELU, p=0.1), **over})


def block(**over):
    return B.make_block_norm_desc(**{**dict(T=40, D=64, post=1, pre=2, gate_rows=10, p=0.1), **over})


@pytest.mark.parametrize("over,code", [
    (dict(T=0), -1), (dict(D=-3), -1), (dict(N=0), -1), (dict(dtype=2), -1), (dict(act=4), -1), (dict(act=-1), -1), (dict(p=-0.1), -1), (dict(p=1.5), -1),
    (dict(p=float("nan")), -1), (dict(alpha=float("inf")), -1), (dict(alpha=float("nan")), -1), (dict(site=1 << 24), -1), (dict(ld_x=63), -1), (dict(ld_w=10), -1),
    (dict(ld_r=47), -1), (dict(ld_x=-1), -1), (dict(T=(1 << 22) + 1), -2), (dict(D=(1 << 18) + 1), -2), (dict(N=1 << 19), -2), (dict(ld_x=(1 << 20) + 1), -2),
    (dict(T=1 << 22, N=1 << 18), -2)])
def test_linear_descriptors(over, code):
    d = linear(**over)
    for op in (B.LINEAR_FWD, B.LINEAR_BWD):
        n = ctypes.c_size_t()
        refused(B.lib().cac_linear_workspace_size(d, op, ctypes.byref(n)), code)
        refused(Linear.call(d, op, ws_bytes=1 << 40), code)


@pytest.mark.parametrize("over,code", [
    (dict(T=0), -1), (dict(D=0), -1), (dict(dtype=-1), -1), (dict(post=3), -1), (dict(pre=-1), -1), (dict(gate_rows=-1), -1), (dict(eps_post=-1e-5), -1),
    (dict(eps_pre=float("nan")), -1), (dict(eps_pre=float("inf")), -1), (dict(p=2.0), -1), (dict(site=1 << 30), -1), (dict(ld_f=60), -1), (dict(ld_r=1), -1),
    (dict(alpha=float("nan")), -1), (dict(D=(1 << 14) + 1), -2), (dict(T=(1 << 28) + 1), -2), (dict(ld_f=1 << 21), -2)])
def test_norm_descriptors(over, code):
    d = block(**over)
    for op in (B.BLOCK_NORM_FWD, B.BLOCK_NORM_BWD):
        n = ctypes.c_size_t()
        refused(B.lib().cac_block_norm_workspace_size(d, op, ctypes.byref(n)), code)
        refused(Norm.call(d, op, ws_bytes=1 << 40), code)


@pytest.mark.parametrize("over,code", [
    (dict(rows=0), -1), (dict(cols=0), -1), (dict(dtype=9), -1), (dict(ld_x=5), -1), (dict(ld_r=-5), -1), (dict(p=1.01), -1), (dict(p=float("nan")), -1),
    (dict(site=1 << 24), -1), (dict(alpha=float("inf")), -1), (dict(rows=(1 << 31) - 1, cols=1 << 13), -2), (dict(cols=(1 << 30) + 1), -2)])
def test_dropout_descriptors(over, code):
    d = B.make_dropout_desc(**{**dict(rows=10, cols=64, p=0.1), **over})
    a = addresses(("X", "R", "rng", "Y"))
    refused(B.lib().cac_dropout(d, a["X"], a["R"], a["rng"], a["Y"], None), code)


def test_sizes_of_descriptors_ops_and_null():
    L, n = B.lib(), ctypes.c_size_t()
    for make, size, plan in ((linear, L.cac_linear_workspace_size, L.cac_linear_describe_plan),
                             (block, L.cac_block_norm_workspace_size, L.cac_block_norm_describe_plan)):
        d = make()
        buf = ctypes.create_string_buffer(300)
        for op in (0, 1):
            assert size(d, op, ctypes.byref(n)) == B.CAC_OK and plan(d, op, buf, 300) == B.CAC_OK and len(buf.value) > 10
            assert plan(d, op, buf, 5) == B.CAC_OK and len(buf.value) == 4
            refused(size(d, op, None), -1)
            refused(plan(d, op, None, 10), -1)
            refused(plan(d, op, buf, 0), -1)
        refused(size(d, 2, ctypes.byref(n)), -1, "op")
        refused(size(None, 0, ctypes.byref(n)), -1, "descriptor")
        d.size -= 4
        refused(size(d, 0, ctypes.byref(n)), -1, "desc.size")
    d = B.make_dropout_desc(3, 3)
    d.size = 0
    refused(L.cac_dropout(d, 64, None, None, 128, None), -1, "desc.size")
    refused(L.cac_dropout(None, 64, None, None, 128, None), -1, "descriptor")


@pytest.mark.parametrize("dtype", ALL)
def test_pointers_that_are_missing_or_not_aligned(dtype):
    for op, names, need in ((B.LINEAR_FWD, Linear.fwd, ("X", "W", "b", "rng", "Y")), (B.LINEAR_BWD, Linear.bwd, ("X", "W", "b", "dY", "rng"))):
        d = linear(dtype=dtype)
        for n in need:
            refused(Linear.call(d, op, **{n: None}), -1, n)
        for n in names:
            refused(Linear.call(d, op, **{n: 64 * MB + 8}), -4, n)
        refused(Linear.call(linear(dtype=dtype, T=400, D=63), op, ws=None), -3)
        refused(Linear.call(linear(dtype=dtype, T=400, D=63), op, ws_bytes=16), -3)
        refused(Linear.call(linear(dtype=dtype, T=400, D=63), op, ws=(1 << 33) + 4), -4)
    refused(Linear.call(linear(dtype=dtype), B.LINEAR_BWD, dX=None, dW=None, db=None), -1, "nothing")
    d = block(dtype=dtype)
    for op, names, need in ((B.BLOCK_NORM_FWD, Norm.fwd, ("F", "gate", "rng", "H")), (B.BLOCK_NORM_BWD, Norm.bwd, ("F", "S", "gate", "dH", "rng"))):
        for n in need:
            refused(Norm.call(d, op, **{n: None}), -1, n)
        for n in names:
            refused(Norm.call(d, op, **{n: 64 * MB + 4}), -4, n)
    refused(Norm.call(d, B.BLOCK_NORM_BWD, ws_bytes=0), -3)
    refused(Norm.call(d, B.BLOCK_NORM_BWD, **{n: None for n in Norm.bwd[9:]}), -1, "nothing")
    refused(Norm.call(block(pre=0, post=0, gate_rows=0), B.BLOCK_NORM_FWD, S=None, H=None, gate=None, w_post=None, b_post=None, w_pre=None, b_pre=None), -1, "nothing")
    a = addresses(("X", "R", "rng", "Y"))
    d = B.make_dropout_desc(10, 64, dtype=dtype, p=0.1)
    for n in ("X", "rng", "Y"):
        refused(B.lib().cac_dropout(d, *({**a, n: None}[k] for k in ("X", "R", "rng", "Y")), None), -1, n)
    for n in a:
        refused(B.lib().cac_dropout(d, *({**a, n: 64 * MB + 2}[k] for k in ("X", "R", "rng", "Y")), None), -4, n)


def test_arguments_that_the_descriptor_has_no_place_for():
    off = dict(gate=None, w_post=None, b_post=None, dgate=None, dw_post=None, db_post=None)
    for op, names in ((B.BLOCK_NORM_FWD, ("gate", "w_post", "b_post")), (B.BLOCK_NORM_BWD, ("gate", "w_post", "b_post", "dgate", "dw_post", "db_post"))):
        for n in names:
            refused(Norm.call(block(post=0, gate_rows=0), op, **{**off, n: 64 * MB * 40}), -1, n)
    off = dict(w_pre=None, b_pre=None, H=None, dH=None, dw_pre=None, db_pre=None)
    for op, names in ((B.BLOCK_NORM_FWD, ("w_pre", "b_pre", "H")), (B.BLOCK_NORM_BWD, ("w_pre", "dH", "dw_pre", "db_pre"))):
        for n in names:
            refused(Norm.call(block(pre=0), op, **{**off, n: 64 * MB * 40}), -1, n)
    refused(Norm.call(block(pre=0), B.BLOCK_NORM_BWD, **{**off, "dS": None}), -1, "dS")


@pytest.mark.parametrize("dtype", ALL)
def test_outputs_share_no_memory(dtype):
    """Each output's last 16 bytes over another buffer's first, and the other way round."""
    e = 4 if dtype == B.F32 else 2

    def over(call, d, op, order, sizes, written, ws, need, allowed):
        at = addresses(order)
        for out in written:
            for other in (*order, "ws"):
                if other == out or (other == "ws" and need == 0):
                    continue
                size = need if other == "ws" else sizes[other]
                base = ws if other == "ws" else at[other]
                places = [base + (size - 1) // 16 * 16, base - (sizes[out] - 1) // 16 * 16]
                if (out, other) not in allowed:
                    places.append(base)
                for place in places:
                    if place == base and (out, other) in allowed:
                        continue
                    refused(call(d, op, ws=ws, ws_bytes=need, **{out: place}), -1, "shares memory")

    T, D, N, ws = 41, 64, 48, 1 << 33
    sizes = {"X": T * D * e, "W": N * D * e, "b": N * e, "R": T * N * e, "rng": 16, "Y": T * N * e, "dY": T * N * e, "dX": T * D * e, "dW": N * D * e, "db": N * e}
    d = linear(T=T, D=D, N=N, dtype=dtype)
    for op, order, written, allowed in ((B.LINEAR_FWD, Linear.fwd, ("Y",), {("Y", "R")}), (B.LINEAR_BWD, Linear.bwd, ("dX", "dW", "db"), set())):
        over(Linear.call, d, op, order, sizes, written, ws, B.cac_linear_workspace_size(d, op), allowed)
    refused(Linear.call(linear(T=T, D=D, N=N, dtype=dtype, ld_r=N + 8), B.LINEAR_FWD, Y=addresses(Linear.fwd)["R"]), -1, "shares memory")
    d = block(T=T, D=D, dtype=dtype)
    vec, whole = 4 * D, T * D * e
    sizes = {**{k: vec for k in ("w_post", "b_post", "w_pre", "b_pre", "dw_post", "db_post", "dw_pre", "db_pre")}, "gate": 5 * vec, "dgate": 5 * vec, "rng": 16,
             **{k: whole for k in ("F", "R", "S", "H", "dH", "dS", "dR", "dF")}}
    over(Norm.call, d, B.BLOCK_NORM_FWD, Norm.fwd, sizes, ("S", "H"), ws, 0, {("S", "R")})
    over(Norm.call, d, B.BLOCK_NORM_BWD, Norm.bwd, sizes, Norm.bwd[9:], ws, B.cac_block_norm_workspace_size(d, B.BLOCK_NORM_BWD), {("dR", "dS"), ("dF", "F")})
    order = ("X", "R", "rng", "Y")
    sizes = {"X": T * D * e, "R": T * D * e, "rng": 16, "Y": T * D * e}

    def dropout(d, op, ws, ws_bytes, **o):
        p = {**addresses(order), **o}
        return B.lib().cac_dropout(d, *(p[k] for k in order), None)

    over(dropout, B.make_dropout_desc(T, D, dtype=dtype, p=0.1), 0, order, sizes, ("Y",), ws, 0, {("Y", "X"), ("Y", "R")})


@pytest.mark.parametrize("dtype", ALL)
def test_long_rows_are_read_twice_and_not_written_over(dtype):
    """Above 8192 columns the sums over rows read F and dS again."""
    a = addresses(Norm.bwd)
    d = block(D=8200, dtype=dtype)
    refused(Norm.call(d, B.BLOCK_NORM_BWD, dR=a["dS"]), -1, "dR shares memory with dS")
    refused(Norm.call(d, B.BLOCK_NORM_BWD, dF=a["F"]), -1, "dF shares memory with F")


def test_plans_follow_sizes():
    """Workspaces hold what is packed, the gradient before the activation, and partial sums."""
    assert B.cac_linear_workspace_size(linear(T=4096, D=2048, N=2048), B.LINEAR_FWD) == 0
    odd = B.cac_linear_workspace_size(linear(T=4096, D=2047, N=2048), B.LINEAR_FWD)
    assert odd == 2 * (4096 + 2048) * 2048
    grad = B.cac_linear_workspace_size(linear(T=4096, D=2048, N=2048), B.LINEAR_BWD)
    assert grad >= 2 * 4096 * 2048
    assert B.cac_block_norm_workspace_size(block(T=1, D=2048, gate_rows=0), B.BLOCK_NORM_BWD) == 0
