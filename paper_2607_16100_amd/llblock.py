"""Python binding of the block C ABI (``include/llblock.h``), same library as
``llcoll``.

Argument marshalling only, as in ``llcoll``: every function has the C name,
takes the same arguments (device pointers and streams as integers, 0 or None
for NULL) and returns the C status code.  ``moe`` and ``optim`` hold the
torch-level calls.
"""
from __future__ import annotations

import ctypes

from . import llcoll as ll
from .llmoe import LLLinearDesc

LL_BLOCK = 128
LL_NORM_MAX_FEATURES = 16384
LL_ADAMW_WORKSPACE = 64
LL_ADAMW_FLOOR = 0x100

_vp, _sz, _i, _u32, _u64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_uint32, ctypes.c_uint64
_f, _d = ctypes.c_float, ctypes.c_double


class LLNormDesc(ctypes.Structure):
    """ll_norm_desc (include/llblock.h)."""
    _fields_ = [("size", _u32), ("dt", _i), ("wdt", _i), ("eps", _f), ("scale", _f), ("rows", _sz), ("features", _sz),
                ("ldy", _sz), ("ldx", _sz), ("ldr", _sz), ("ldh", _sz), ("ldq", _sz), ("lds", _sz), ("ldd", _sz),
                ("ldo", _sz), ("lddy", _sz)]


class LLAdamwTensor(ctypes.Structure):
    """ll_adamw_tensor (include/llblock.h)."""
    _fields_ = [("param", _vp), ("grad", _vp), ("master", _vp), ("m", _vp), ("v", _vp), ("m_scales", _vp),
                ("v_scales", _vp), ("n", _sz), ("at", _u64), ("dt", _i), ("gdt", _i)]


class LLAdamwDesc(ctypes.Structure):
    """ll_adamw_desc (include/llblock.h)."""
    _fields_ = [("size", _u32), ("bits", ctypes.c_int32), ("lr", _d), ("beta1", _d), ("beta2", _d), ("eps", _d),
                ("decay", _d), ("seed", _u32)]


NORM_DESC_SIZE = ctypes.sizeof(LLNormDesc)
ADAMW_DESC_SIZE = ctypes.sizeof(LLAdamwDesc)
_L, _N = ctypes.POINTER(LLLinearDesc), ctypes.POINTER(LLNormDesc)
_A, _T = ctypes.POINTER(LLAdamwDesc), ctypes.POINTER(LLAdamwTensor)

# name -> argtypes (every function returns a status)
_SIGS = {
    "ll_quantise": [_vp, _sz, _sz, _vp, _sz, _i, _i, _vp, _sz, _vp, _sz, _vp],
    "ll_quantise_weight": [_vp, _sz, _sz, _i, _sz, _sz, _i, _i, _vp, _sz, _sz, _vp, _sz, _sz, _vp],
    "ll_linear8": [_L, _vp, _vp, _sz, _vp, _vp, _sz, _sz, _vp, _vp, _vp, _vp, _vp, _sz, _vp],
    "ll_linear8_bytes": [_L, ctypes.POINTER(_sz)],
    "ll_norm_desc_init": [_N, _i, _i, _sz, _sz, _f, _f],
    "ll_norm": [_N, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp],
    "ll_norm_grad": [_N, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _u32, _vp, _sz, _vp],
    "ll_norm_bytes": [_N, ctypes.POINTER(_sz)],
    "ll_adamw": [_A, _T, _sz, _vp, _vp, _vp, _vp, _sz, _vp],
}

_lib = ll.library()
for _name, _args in _SIGS.items():
    _fn = getattr(_lib, _name)
    _fn.restype = _i
    _fn.argtypes = _args


def exported_symbols():
    return list(_SIGS)


def norm_desc(dt: int, wdt: int, rows: int, features: int, eps: float, scale: float, **fields) -> LLNormDesc:
    """An ll_norm_desc with contiguous rows, then `fields` set."""
    d = LLNormDesc()
    ll.check(_lib.ll_norm_desc_init(ctypes.byref(d), dt, wdt, rows, features, eps, scale), "ll_norm_desc_init")
    for k, v in fields.items():
        if k not in ("ldy", "ldx", "ldr", "ldh", "ldq", "lds", "ldd", "ldo", "lddy", "size"):
            raise TypeError(f"unknown field {k}")
        setattr(d, k, v)
    return d


def ll_quantise(x, ldx, rows, end, features, dt, act, q, ldq, scales, lds, stream):
    return _lib.ll_quantise(x, ldx, rows, end, features, dt, act, q, ldq, scales, lds, stream)


def ll_quantise_weight(w, ldw, wstride, groups, out, in_, dt, transpose, q, ldq, qstride, scales, lds, sstride, stream):
    return _lib.ll_quantise_weight(w, ldw, wstride, groups, out, in_, dt, transpose, q, ldq, qstride, scales, lds,
                                   sstride, stream)


def ll_linear8(d, x, xs, ldxs, w, ws, ldws, wsstride, bias, residual, y, z, workspace, workspace_bytes, stream):
    return _lib.ll_linear8(ctypes.byref(d), x, xs, ldxs, w, ws, ldws, wsstride, bias, residual, y, z, workspace,
                           workspace_bytes, stream)


def ll_linear8_bytes(d: LLLinearDesc):
    """(status, workspace bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.ll_linear8_bytes(ctypes.byref(d), ctypes.byref(out))
    return st, out.value


def ll_norm(d, y, x, gate, post, weight, r, h, q, scales, stream):
    return _lib.ll_norm(ctypes.byref(d), y, x, gate, post, weight, r, h, q, scales, stream)


def ll_norm_grad(d, dh, r, dr, y, gate, post, weight, dr_out, dy, dgate, dweight, dpost, flags, workspace,
                 workspace_bytes, stream):
    return _lib.ll_norm_grad(ctypes.byref(d), dh, r, dr, y, gate, post, weight, dr_out, dy, dgate, dweight, dpost,
                             flags, workspace, workspace_bytes, stream)


def ll_norm_bytes(d: LLNormDesc):
    """(status, workspace bytes)."""
    out = ctypes.c_size_t(0)
    st = _lib.ll_norm_bytes(ctypes.byref(d), ctypes.byref(out))
    return st, out.value


def ll_adamw(d, tensors, count, step, lr_ptr, grad_scale, workspace, workspace_bytes, stream):
    """``tensors``: a ctypes array of LLAdamwTensor, or None."""
    return _lib.ll_adamw(ctypes.byref(d), tensors, count, step, lr_ptr, grad_scale, workspace, workspace_bytes, stream)
