"""Python binding of the expert-layer C ABI (``include/llmoe.h``), same library
as ``llcoll``.

Argument marshalling only, as in ``llcoll``: every function has the C name,
takes the same arguments (device pointers and streams as integers, 0 or None
for NULL) and returns the C status code.  ``moe`` holds the torch-level calls.
"""
from __future__ import annotations

import ctypes

from . import llcoll as ll

LL_SCORE_SOFTMAX, LL_SCORE_SIGMOID = 0, 1
LL_ACT_NONE, LL_ACT_RELU, LL_ACT_GELU, LL_ACT_SILU, LL_ACT_SWIGLU, LL_ACT_GEGLU = range(6)
LL_LINEAR_FORWARD, LL_LINEAR_GRAD_X, LL_LINEAR_GRAD_W = range(3)
LL_GRAD_F32, LL_GRAD_ADD = 0x1, 0x2
LL_MOE_MAX_EXPERTS, LL_MOE_MAX_K = 1024, 32

SCORES = {"softmax": LL_SCORE_SOFTMAX, "sigmoid": LL_SCORE_SIGMOID}
ACTS = {"none": LL_ACT_NONE, "relu": LL_ACT_RELU, "gelu": LL_ACT_GELU, "silu": LL_ACT_SILU,
        "swiglu": LL_ACT_SWIGLU, "geglu": LL_ACT_GEGLU}
GATED = ("swiglu", "geglu")

_vp, _sz, _i, _u32, _f = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_uint32, ctypes.c_float


class LLLinearDesc(ctypes.Structure):
    """ll_linear_desc (include/llmoe.h)."""
    _fields_ = [("size", _u32), ("dt", _i), ("act", _i), ("groups", _i), ("rows", _sz), ("in_", _sz), ("out", _sz),
                ("offsets", _vp), ("ldx", _sz), ("ldw", _sz), ("wstride", _sz), ("ldy", _sz), ("ldz", _sz),
                ("ldr", _sz)]


DESC_SIZE = ctypes.sizeof(LLLinearDesc)
_D = ctypes.POINTER(LLLinearDesc)

# name -> argtypes (every function returns a status)
_SIGS = {
    "ll_moe_route": [_vp, _sz, _sz, _i, _i, _i, _vp, _i, _i, _f, _vp, _vp, _vp],
    "ll_moe_route_grad": [_vp, _sz, _sz, _i, _i, _i, _i, _i, _f, _vp, _vp, _vp, _sz, _vp],
    "ll_moe_dispatch_bytes": [_sz, _i, _i, ctypes.POINTER(_sz)],
    "ll_moe_dispatch": [_vp, _sz, _i, _i, _i, _vp, _sz, _sz, _i, _vp, _vp, _vp, _vp, _sz, _vp, _sz, _vp],
    "ll_moe_combine": [_vp, _sz, _sz, _vp, _vp, _vp, _sz, _sz, _i, _sz, _i, _vp, _sz, _vp],
    "ll_moe_combine_grad": [_vp, _sz, _vp, _sz, _sz, _vp, _vp, _sz, _i, _sz, _i, _vp, _sz, _vp, _vp],
    "ll_linear_desc_init": [_D, _i, _i, _i, _sz, _sz, _sz],
    "ll_linear_bytes": [_D, _i, ctypes.POINTER(_sz)],
    "ll_linear": [_D, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "ll_linear_grad_x": [_D, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "ll_linear_grad_w": [_D, _vp, _vp, _vp, _vp, _u32, _vp, _sz, _vp],
    "ll_act_grad": [_vp, _sz, _vp, _sz, _sz, _sz, _i, _i, _vp, _sz, _vp],
}

_lib = ll.library()
for _name, _args in _SIGS.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _i
    _fn.argtypes = _args


def exported_symbols():
    return list(_SIGS)


def desc(dt: int, act: int, groups: int, rows: int, in_: int, out: int, **fields) -> LLLinearDesc:
    """An ll_linear_desc with contiguous rows, then `fields` set."""
    d = LLLinearDesc()
    ll.check(_lib.ll_linear_desc_init(ctypes.byref(d), dt, act, groups, rows, in_, out), "ll_linear_desc_init")
    for k, v in fields.items():
        if k not in ("offsets", "ldx", "ldw", "wstride", "ldy", "ldz", "ldr", "size"):
            raise TypeError(f"unknown field {k}")
        setattr(d, k, v)
    return d


def ll_moe_route(logits, ld, tokens, experts, k, dt, bias, score, normalise, scale, ids, weights, stream):
    return _lib.ll_moe_route(logits, ld, tokens, experts, k, dt, bias, score, normalise, scale, ids, weights, stream)


def ll_moe_route_grad(logits, ld, tokens, experts, k, dt, score, normalise, scale, ids, dweights, dlogits, ldd,
                      stream):
    return _lib.ll_moe_route_grad(logits, ld, tokens, experts, k, dt, score, normalise, scale, ids, dweights,
                                  dlogits, ldd, stream)


def ll_moe_dispatch_bytes(tokens: int, k: int, experts: int):
    """(status, workspace bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.ll_moe_dispatch_bytes(tokens, k, experts, ctypes.byref(out))
    return st, out.value


def ll_moe_dispatch(ids, tokens, k, first, experts, x, ldx, features, dt, offsets, slots, rows, y, ldy, workspace,
                    workspace_bytes, stream):
    return _lib.ll_moe_dispatch(ids, tokens, k, first, experts, x, ldx, features, dt, offsets, slots, rows, y, ldy,
                                workspace, workspace_bytes, stream)


def ll_moe_combine(y, ldy, nrows, rows, weights, residual, ldr, tokens, k, features, dt, out, ldo, stream):
    return _lib.ll_moe_combine(y, ldy, nrows, rows, weights, residual, ldr, tokens, k, features, dt, out, ldo, stream)


def ll_moe_combine_grad(dout, ldd, y, ldy, nrows, rows, weights, tokens, k, features, dt, dy, lddy, dweights, stream):
    return _lib.ll_moe_combine_grad(dout, ldd, y, ldy, nrows, rows, weights, tokens, k, features, dt, dy, lddy,
                                    dweights, stream)


def ll_linear_bytes(d: LLLinearDesc, which: int):
    """(status, workspace bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.ll_linear_bytes(ctypes.byref(d), which, ctypes.byref(out))
    return st, out.value


def ll_linear(d, x, w, bias, residual, y, z, workspace, workspace_bytes, stream):
    return _lib.ll_linear(ctypes.byref(d), x, w, bias, residual, y, z, workspace, workspace_bytes, stream)


def ll_linear_grad_x(d, dz, w, z, dx, workspace, workspace_bytes, stream):
    return _lib.ll_linear_grad_x(ctypes.byref(d), dz, w, z, dx, workspace, workspace_bytes, stream)


def ll_linear_grad_w(d, dz, x, dw, dbias, flags, workspace, workspace_bytes, stream):
    return _lib.ll_linear_grad_w(ctypes.byref(d), dz, x, dw, dbias, flags, workspace, workspace_bytes, stream)


def ll_act_grad(dy, lddy, z, ldz, rows, features, dt, act, dz, lddz, stream):
    return _lib.ll_act_grad(dy, lddy, z, ldz, rows, features, dt, act, dz, lddz, stream)
