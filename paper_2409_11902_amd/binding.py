"""ctypes binding of libcac.so: argument marshalling only.

Function names and argument order follow include/cac.h.  Tensors are torch
tensors on the GPU (torch is used for device memory and streams, nothing else);
every computation happens inside the library's HIP kernels.  A missing library
is an error: there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

from . import synth

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcac.so")

CAC_OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE_TOO_SMALL, ERR_ALIGNMENT, ERR_LAUNCH_FAILED = -1, -2, -3, -4, -5
F32, BF16 = 0, 1
DW_INFLATE, DW_REDUCED_K, DW_AUTO = 0, 1, 2
EDGE_CEIL_VALID, EDGE_FLOOR_DROP = 0, 1
POOL_MEAN, POOL_MAX = 0, 1
(OP_FWD_AND_COMPRESS, OP_BWD_WEIGHT_COMPRESSED, OP_BWD_DATA, OP_COMPRESS, OP_BWD_BIAS, OP_GRAD_COSINE,
 OP_BWD_WEIGHT_AND_DATA, OP_BN_BWD) = range(8)

EXPORTS = (
    "cac_version", "cac_last_error", "cac_out_shape", "cac_pooled_shape", "cac_workspace_size", "cac_describe_plan",
    "cac_dw_executed_flops",
    "conv_fwd_and_compress", "cac_compress", "conv_bwd_weight_compressed", "conv_bwd_data", "conv_bwd_bias", "cac_grad_cosine",
    "conv_bwd_weight_and_data", "conv_bwd_weight_compressed_noalloc", "cac_bn_relu_fwd_compress", "cac_bn_bwd_compressed", "cac_probe",
    "cac_loss_workspace_size", "cac_loss_describe_plan", "cac_loss_fwd", "cac_loss_bwd",
    "cac_muon_workspace_size", "cac_muon_describe_plan", "cac_orthogonalise", "cac_muon_step",
    "cac_dropout", "cac_linear_workspace_size", "cac_linear_describe_plan", "cac_linear_fwd", "cac_linear_bwd",
    "cac_block_norm_workspace_size", "cac_block_norm_describe_plan", "cac_block_norm_fwd", "cac_block_norm_bwd",
)
LOSS_FWD, LOSS_BWD = 0, 1
MUON_ORTHOGONALISE, MUON_STEP = 0, 1
LINEAR_FWD, LINEAR_BWD = 0, 1
BLOCK_NORM_FWD, BLOCK_NORM_BWD = 0, 1
ACT_NONE, ACT_RELU, ACT_GELU, ACT_SILU = range(4)
NORM_NONE, NORM_RMS, NORM_LAYER = range(3)
PROBE_MFMA, PROBE_COPY, PROBE_READ, PROBE_MFMA_16X16, PROBE_MFMA_1WAVE = 0, 1, 2, 3, 4
NOALLOC_SCRATCH_BYTES = 40 << 20


class cac_desc(ctypes.Structure):
    _fields_ = [("size", ctypes.c_uint32)] + [
        (n, ctypes.c_int32) for n in (
            "N", "C_in", "C_out", "H", "W", "R", "S", "stride_h", "stride_w", "pad_h", "pad_w",
            "pool_kh", "pool_kw", "edge_mode", "dtype", "has_bias", "pool_mode", "dw_algo")
    ]


class cac_loss_desc(ctypes.Structure):
    _fields_ = [("size", ctypes.c_uint32)] + [
        (n, ctypes.c_int32) for n in ("T", "D", "V", "ld_h", "ld_w", "dtype", "has_bias", "ignore_index")
    ]


class cac_muon_desc(ctypes.Structure):
    _fields_ = [("size", ctypes.c_uint32)] + [
        (n, ctypes.c_int32) for n in ("batch", "rows", "cols", "dtype", "grad_dtype", "steps", "nesterov")
    ]


class cac_dropout_desc(ctypes.Structure):
    _fields_ = [("size", ctypes.c_uint32)] + [(n, ctypes.c_int32) for n in ("rows", "cols", "ld_x", "ld_r", "dtype")] + [
        ("alpha", ctypes.c_float), ("drop_p", ctypes.c_float), ("site", ctypes.c_uint32)]


class cac_linear_desc(ctypes.Structure):
    _fields_ = [("size", ctypes.c_uint32)] + [
        (n, ctypes.c_int32) for n in ("T", "D", "N", "ld_x", "ld_w", "ld_r", "dtype", "has_bias", "act")
    ] + [("alpha", ctypes.c_float), ("drop_p", ctypes.c_float), ("site", ctypes.c_uint32)]


class cac_block_norm_desc(ctypes.Structure):
    _fields_ = [("size", ctypes.c_uint32)] + [
        (n, ctypes.c_int32) for n in ("T", "D", "ld_f", "ld_r", "dtype", "post", "pre", "gate_rows")
    ] + [(n, ctypes.c_float) for n in ("eps_post", "eps_pre", "alpha", "drop_p")] + [("site", ctypes.c_uint32)]


class CacError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"cac error {code}: {msg}")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded native library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2409_11902_amd.build` "
                "(there is no fallback implementation)")
        L = ctypes.CDLL(LIB_PATH)
        L.cac_version.restype = ctypes.c_int
        L.cac_last_error.restype = ctypes.c_char_p
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        dp = ctypes.POINTER(cac_desc)
        ip = ctypes.POINTER(ctypes.c_int32)
        szp = ctypes.POINTER(ctypes.c_size_t)
        L.cac_out_shape.argtypes = [dp, ip, ip]
        L.cac_pooled_shape.argtypes = [dp, ip, ip, szp, szp]
        L.cac_workspace_size.argtypes = [dp, ctypes.c_int, szp]
        L.cac_describe_plan.argtypes = [dp, ctypes.c_int, ctypes.c_char_p, sz]
        L.cac_dw_executed_flops.argtypes = [dp, ctypes.POINTER(ctypes.c_uint64)]
        L.conv_fwd_and_compress.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.cac_compress.argtypes = [dp, vp, vp, vp]
        L.conv_bwd_weight_compressed.argtypes = [dp, vp, vp, vp, vp, sz, vp]
        L.conv_bwd_weight_compressed_noalloc.argtypes = [dp, vp, vp, vp, vp]
        L.conv_bwd_data.argtypes = [dp, vp, vp, vp, vp, sz, vp]
        L.conv_bwd_weight_and_data.argtypes = [dp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.conv_bwd_bias.argtypes = [dp, vp, vp, vp]
        L.cac_probe.argtypes = [ctypes.c_int, vp, vp, sz, ctypes.c_int, vp]
        L.cac_bn_relu_fwd_compress.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp]
        L.cac_bn_bwd_compressed.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.cac_grad_cosine.argtypes = [dp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        lp, mp, fl = ctypes.POINTER(cac_loss_desc), ctypes.POINTER(cac_muon_desc), ctypes.c_float
        L.cac_loss_workspace_size.argtypes = [lp, ctypes.c_int, szp]
        L.cac_loss_describe_plan.argtypes = [lp, ctypes.c_int, ctypes.c_char_p, sz]
        L.cac_loss_fwd.argtypes = [lp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.cac_loss_bwd.argtypes = [lp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.cac_muon_workspace_size.argtypes = [mp, ctypes.c_int, szp]
        L.cac_muon_describe_plan.argtypes = [mp, ctypes.c_int, ctypes.c_char_p, sz]
        L.cac_orthogonalise.argtypes = [mp, vp, vp, vp, sz, vp]
        L.cac_muon_step.argtypes = [mp, vp, vp, vp, fl, fl, fl, vp, sz, vp]
        odp, idp, ndp = ctypes.POINTER(cac_dropout_desc), ctypes.POINTER(cac_linear_desc), ctypes.POINTER(cac_block_norm_desc)
        L.cac_dropout.argtypes = [odp] + [vp] * 5
        L.cac_linear_workspace_size.argtypes = [idp, ctypes.c_int, szp]
        L.cac_linear_describe_plan.argtypes = [idp, ctypes.c_int, ctypes.c_char_p, sz]
        L.cac_linear_fwd.argtypes = [idp] + [vp] * 7 + [sz, vp]
        L.cac_linear_bwd.argtypes = [idp] + [vp] * 9 + [sz, vp]
        L.cac_block_norm_workspace_size.argtypes = [ndp, ctypes.c_int, szp]
        L.cac_block_norm_describe_plan.argtypes = [ndp, ctypes.c_int, ctypes.c_char_p, sz]
        L.cac_block_norm_fwd.argtypes = [ndp] + [vp] * 11
        L.cac_block_norm_bwd.argtypes = [ndp] + [vp] * 17 + [sz, vp]
        for n in EXPORTS[2:]:
            getattr(L, n).restype = ctypes.c_int
        _lib = L
    return _lib


def _check(rc: int):
    if rc != CAC_OK:
        raise CacError(rc, lib().cac_last_error().decode())


def make_desc(N, C_in, C_out, H, W, R, S, stride_h=1, stride_w=1, pad_h=0, pad_w=0, pool_kh=2, pool_kw=2,
              edge_mode=EDGE_CEIL_VALID, dtype=BF16, has_bias=1, pool_mode=POOL_MEAN, dw_algo=DW_INFLATE) -> cac_desc:
    return cac_desc(ctypes.sizeof(cac_desc), N, C_in, C_out, H, W, R, S, stride_h, stride_w, pad_h, pad_w,
                    pool_kh, pool_kw, edge_mode, dtype, has_bias, pool_mode, dw_algo)


def make_loss_desc(T, D, V, dtype=BF16, has_bias=0, ignore_index=-100, ld_h=0, ld_w=0) -> cac_loss_desc:
    return cac_loss_desc(ctypes.sizeof(cac_loss_desc), T, D, V, ld_h, ld_w, dtype, has_bias, ignore_index)


def make_muon_desc(rows, cols, batch=1, dtype=F32, grad_dtype=F32, steps=5, nesterov=1) -> cac_muon_desc:
    return cac_muon_desc(ctypes.sizeof(cac_muon_desc), batch, rows, cols, dtype, grad_dtype, steps, nesterov)


def make_dropout_desc(rows, cols, dtype=BF16, p=0.0, alpha=1.0, site=0, ld_x=0, ld_r=0) -> cac_dropout_desc:
    return cac_dropout_desc(ctypes.sizeof(cac_dropout_desc), rows, cols, ld_x, ld_r, dtype, alpha, p, site)


def make_linear_desc(T, D, N, dtype=BF16, has_bias=0, act=ACT_NONE, alpha=1.0, p=0.0, site=0, ld_x=0, ld_w=0, ld_r=0) -> cac_linear_desc:
    return cac_linear_desc(ctypes.sizeof(cac_linear_desc), T, D, N, ld_x, ld_w, ld_r, dtype, has_bias, act, alpha, p, site)


def make_block_norm_desc(T, D, dtype=BF16, post=NORM_NONE, pre=NORM_RMS, gate_rows=0, eps_post=1e-5, eps_pre=1e-5, alpha=1.0, p=0.0, site=0,
                         ld_f=0, ld_r=0) -> cac_block_norm_desc:
    return cac_block_norm_desc(ctypes.sizeof(cac_block_norm_desc), T, D, ld_f, ld_r, dtype, post, pre, gate_rows, eps_post, eps_pre, alpha, p, site)


def desc_from_spec(spec: synth.LayerSpec, has_bias: int = 1, **over) -> cac_desc:
    kw = dict(N=spec.N, C_in=spec.C, C_out=spec.K, H=spec.H, W=spec.W, R=spec.R, S=spec.S,
              stride_h=spec.stride, stride_w=spec.stride, pad_h=spec.pad, pad_w=spec.pad,
              pool_kh=spec.k, pool_kw=spec.k, dtype=F32 if spec.dtype == synth.F32 else BF16,
              has_bias=has_bias)
    kw.update(over)
    return make_desc(**kw)


def cac_version() -> int:
    return lib().cac_version()


def cac_out_shape(d: cac_desc):
    p, q = ctypes.c_int32(), ctypes.c_int32()
    _check(lib().cac_out_shape(ctypes.byref(d), ctypes.byref(p), ctypes.byref(q)))
    return p.value, q.value


def cac_pooled_shape(d: cac_desc):
    """(Hp, Wp, z_bytes, x_bytes)"""
    hp, wp = ctypes.c_int32(), ctypes.c_int32()
    zb, xb = ctypes.c_size_t(), ctypes.c_size_t()
    _check(lib().cac_pooled_shape(ctypes.byref(d), ctypes.byref(hp), ctypes.byref(wp), ctypes.byref(zb),
                                  ctypes.byref(xb)))
    return hp.value, wp.value, zb.value, xb.value


def cac_workspace_size(d: cac_desc, op: int) -> int:
    b = ctypes.c_size_t()
    _check(lib().cac_workspace_size(ctypes.byref(d), op, ctypes.byref(b)))
    return b.value


def cac_describe_plan(d: cac_desc, op: int) -> str:
    buf = ctypes.create_string_buffer(2048)
    _check(lib().cac_describe_plan(ctypes.byref(d), op, buf, len(buf)))
    return buf.value.decode()


def dw_rk_executed_flops(d: cac_desc) -> int:
    f = ctypes.c_uint64()
    _check(lib().cac_dw_executed_flops(ctypes.byref(d), ctypes.byref(f)))
    return f.value


# The marshalling of a call costs as much as a third of a launch, so it does no more than it must: pointers go as integers (the
# argument types above take them, None as null), the descriptor as it is, the stream's handle without a stream object around it.

def _ptr(t):
    return None if t is None else t.data_ptr()


_torch = None


def _stream(stream):
    global _torch
    if stream is not None:
        return stream.cuda_stream
    if _torch is None:
        import torch
        _torch = torch
    if _torch.cuda.is_initialized():
        c = _torch._C
        try:
            return c._cuda_getCurrentRawStream(c._cuda_getDevice())
        except AttributeError:
            pass
    return _torch.cuda.current_stream().cuda_stream


def _ws(ws):
    return (None, 0) if ws is None else (ws.data_ptr(), ws.nbytes)


def conv_fwd_and_compress(d, X, W, b, Y, Z, ws=None, stream=None):
    _check((_lib or lib()).conv_fwd_and_compress(d, _ptr(X), _ptr(W), _ptr(b), _ptr(Y), _ptr(Z), *_ws(ws), _stream(stream)))


def cac_compress(d, X, Z, stream=None):
    _check((_lib or lib()).cac_compress(d, _ptr(X), _ptr(Z), _stream(stream)))


def conv_bwd_weight_compressed(d, Z, dY, dW, ws=None, stream=None):
    _check((_lib or lib()).conv_bwd_weight_compressed(d, _ptr(Z), _ptr(dY), _ptr(dW), *_ws(ws), _stream(stream)))


def conv_bwd_weight_compressed_noalloc(d, Z, dY, dW, stream=None):
    _check((_lib or lib()).conv_bwd_weight_compressed_noalloc(d, _ptr(Z), _ptr(dY), _ptr(dW), _stream(stream)))


def conv_bwd_data(d, W, dY, dX, ws=None, stream=None):
    _check((_lib or lib()).conv_bwd_data(d, _ptr(W), _ptr(dY), _ptr(dX), *_ws(ws), _stream(stream)))


def conv_bwd_weight_and_data(d, Z, W, dY, dW, dX, ws=None, stream=None):
    _check((_lib or lib()).conv_bwd_weight_and_data(d, _ptr(Z), _ptr(W), _ptr(dY), _ptr(dW), _ptr(dX), *_ws(ws), _stream(stream)))


def cac_bn_relu_fwd_compress(d, Y, scale, shift, X_next, Z_next, Z_in=None, stream=None):
    _check((_lib or lib()).cac_bn_relu_fwd_compress(d, _ptr(Y), _ptr(scale), _ptr(shift), _ptr(X_next), _ptr(Z_next), _ptr(Z_in),
                                                    _stream(stream)))


def cac_bn_bwd_compressed(d, Z_in, dY, mean, invstd, gamma, dgamma, dbeta, dX, ws=None, stream=None):
    _check((_lib or lib()).cac_bn_bwd_compressed(d, _ptr(Z_in), _ptr(dY), _ptr(mean), _ptr(invstd), _ptr(gamma), _ptr(dgamma),
                                                 _ptr(dbeta), _ptr(dX), *_ws(ws), _stream(stream)))


def cac_probe(kind, src, dst, nbytes, iters=0, stream=None):
    _check((_lib or lib()).cac_probe(kind, _ptr(src), _ptr(dst), nbytes, iters, _stream(stream)))


def conv_bwd_bias(d, dY, db, stream=None):
    _check((_lib or lib()).conv_bwd_bias(d, _ptr(dY), _ptr(db), _stream(stream)))


def cac_grad_cosine(d, dW_a, dW_b, out, ws=None, stream=None):
    _check((_lib or lib()).cac_grad_cosine(d, _ptr(dW_a), _ptr(dW_b), _ptr(out), *_ws(ws), _stream(stream)))


def _size_of(fn, d, op) -> int:
    n = ctypes.c_size_t()
    _check(fn(ctypes.byref(d), op, ctypes.byref(n)))
    return n.value


def _plan_of(fn, d, op) -> str:
    buf = ctypes.create_string_buffer(2048)
    _check(fn(ctypes.byref(d), op, buf, len(buf)))
    return buf.value.decode()


def cac_loss_workspace_size(d: cac_loss_desc, op: int) -> int:
    return _size_of(lib().cac_loss_workspace_size, d, op)


def cac_loss_describe_plan(d: cac_loss_desc, op: int) -> str:
    return _plan_of(lib().cac_loss_describe_plan, d, op)


def cac_loss_fwd(d, H, W, b, labels, loss, lse, ws=None, stream=None):
    _check((_lib or lib()).cac_loss_fwd(d, _ptr(H), _ptr(W), _ptr(b), _ptr(labels), _ptr(loss), _ptr(lse), *_ws(ws), _stream(stream)))


def cac_loss_bwd(d, H, W, b, labels, lse, gloss, dH, dW, db, ws=None, stream=None):
    _check((_lib or lib()).cac_loss_bwd(d, _ptr(H), _ptr(W), _ptr(b), _ptr(labels), _ptr(lse), _ptr(gloss), _ptr(dH), _ptr(dW), _ptr(db),
                                        *_ws(ws), _stream(stream)))


def cac_muon_workspace_size(d: cac_muon_desc, op: int) -> int:
    return _size_of(lib().cac_muon_workspace_size, d, op)


def cac_muon_describe_plan(d: cac_muon_desc, op: int) -> str:
    return _plan_of(lib().cac_muon_describe_plan, d, op)


def cac_orthogonalise(d, G, O, ws=None, stream=None):
    _check((_lib or lib()).cac_orthogonalise(d, _ptr(G), _ptr(O), *_ws(ws), _stream(stream)))


def cac_muon_step(d, G, M, W, momentum, keep, lr, ws=None, stream=None):
    _check((_lib or lib()).cac_muon_step(d, _ptr(G), _ptr(M), _ptr(W), momentum, keep, lr, *_ws(ws), _stream(stream)))


# (pointers in place: a call of _ptr costs as much as data_ptr does, and these have up to 17)

def cac_dropout(d, X, R, rng, Y, stream=None):
    _check((_lib or lib()).cac_dropout(d, None if X is None else X.data_ptr(), None if R is None else R.data_ptr(), None if rng is None else rng.data_ptr(),
                                       None if Y is None else Y.data_ptr(), _stream(stream)))


def cac_linear_workspace_size(d: cac_linear_desc, op: int) -> int:
    return _size_of(lib().cac_linear_workspace_size, d, op)


def cac_linear_describe_plan(d: cac_linear_desc, op: int) -> str:
    return _plan_of(lib().cac_linear_describe_plan, d, op)


def cac_linear_fwd(d, X, W, b, R, rng, Y, ws=None, stream=None):
    _check((_lib or lib()).cac_linear_fwd(
        d, None if X is None else X.data_ptr(), None if W is None else W.data_ptr(), None if b is None else b.data_ptr(),
        None if R is None else R.data_ptr(), None if rng is None else rng.data_ptr(), None if Y is None else Y.data_ptr(), *_ws(ws), _stream(stream)))


def cac_linear_bwd(d, X, W, b, dY, rng, dX, dW, db, ws=None, stream=None):
    _check((_lib or lib()).cac_linear_bwd(
        d, None if X is None else X.data_ptr(), None if W is None else W.data_ptr(), None if b is None else b.data_ptr(),
        None if dY is None else dY.data_ptr(), None if rng is None else rng.data_ptr(), None if dX is None else dX.data_ptr(), None if dW is None else dW.data_ptr(),
        None if db is None else db.data_ptr(), *_ws(ws), _stream(stream)))


def cac_block_norm_workspace_size(d: cac_block_norm_desc, op: int) -> int:
    return _size_of(lib().cac_block_norm_workspace_size, d, op)


def cac_block_norm_describe_plan(d: cac_block_norm_desc, op: int) -> str:
    return _plan_of(lib().cac_block_norm_describe_plan, d, op)


def cac_block_norm_fwd(d, F, R, gate, w_post, b_post, w_pre, b_pre, rng, S, H, stream=None):
    _check((_lib or lib()).cac_block_norm_fwd(
        d, None if F is None else F.data_ptr(), None if R is None else R.data_ptr(), None if gate is None else gate.data_ptr(),
        None if w_post is None else w_post.data_ptr(), None if b_post is None else b_post.data_ptr(),
        None if w_pre is None else w_pre.data_ptr(), None if b_pre is None else b_pre.data_ptr(), None if rng is None else rng.data_ptr(),
        None if S is None else S.data_ptr(), None if H is None else H.data_ptr(), _stream(stream)))


def cac_block_norm_bwd(d, F, S, gate, w_post, b_post, w_pre, dH, dS, rng, dR, dF, dgate, dw_post, db_post, dw_pre, db_pre, ws=None, stream=None):
    given = (F, S, gate, w_post, b_post, w_pre, dH, dS, rng, dR, dF, dgate, dw_post, db_post, dw_pre, db_pre)
    _check((_lib or lib()).cac_block_norm_bwd(d, *[None if t is None else t.data_ptr() for t in given], *_ws(ws), _stream(stream)))


# ---- host <-> device marshalling (type conversion only, no arithmetic)

def to_device(a, dtype: str, device: str = "cuda:0"):
    """float32 host array already rounded to `dtype` -> device tensor of that dtype."""
    import numpy as np
    import torch
    if dtype == synth.F32:
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device)
    bits = synth.bf16_bits(a).view(np.int16)
    return torch.from_numpy(bits).to(device).view(torch.bfloat16)


def to_host(t):
    """device tensor -> float64 host array (bfloat16 widened exactly)."""
    import numpy as np
    import torch
    if t.dtype == torch.bfloat16:
        bits = t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
        return synth.bf16_from_bits(bits).astype(np.float64)
    return t.cpu().numpy().astype(np.float64)
