"""Expert-layer operators on torch tensors (``include/llmoe.h``).

torch provides memory and the stream; every operator runs in the HIP library.
A call checks its tensors, launches on the current stream (or ``stream``) and
returns its outputs, which it allocates unless they are given.  Errors raise
``llcoll.LLError`` with the C status, or ValueError for tensors that do not
fit together or lie on another GPU than the current one.  Matrices have unit
stride along their last dimension; their rows may lie further apart.  Nothing
is recorded for autograd: each operator's gradient is a call of its own, and
inputs that require gradients are refused while gradients are enabled.

What one rank of an expert-parallel layer does between its AllGather and its
ReduceScatter:

    ids, weights = moe.route(logits, k)
    plan = moe.Dispatch(tokens, k, local_experts, hidden, dtype, first=first_local_expert)
    plan.dispatch(ids, x)                                  # plan.x: rows sorted by expert
    h = moe.linear(plan.x, w_up, act="swiglu", offsets=plan.offsets)
    y = moe.linear(h, w_down, offsets=plan.offsets)
    out = moe.combine(y, plan.rows, weights)

``moe.linear`` without offsets is an ordinary dense layer.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import llblock as lb
from . import llcoll as ll
from . import llmoe as lm

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
_DT = {torch.float32: ll.LL_F32, torch.bfloat16: ll.LL_BF16}
# the C functions themselves: llmoe's wrappers add a call and nothing else here
_c = ll.library()
_raw_stream, _device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _stream(stream, dev: int) -> int:
    if stream is None:
        return _raw_stream(dev)
    if stream.device_index != dev:
        raise ValueError("stream: not of the current GPU")
    return stream.cuda_stream


def _new(stream, *shape, dtype, device, make=torch.empty) -> torch.Tensor:
    """Memory of the stream the call runs on: it may be reused there as soon as
    it is released, and nowhere else."""
    if stream is None:
        return make(*shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return make(*shape, dtype=dtype, device=device)


def _dt(t: torch.Tensor) -> int:
    dt = _DT.get(t.dtype)
    if dt is None:
        raise ll.LLError(ll.LL_ERR_UNSUPPORTED, str(t.dtype))
    return dt


def _mat(t: torch.Tensor, name: str, dev: int, rows=None, cols=None, dtype=None) -> int:
    """Checks a matrix on GPU ``dev``, the current one; its leading dimension."""
    shape = t.shape
    if len(shape) != 2 or t.get_device() != dev:
        raise ValueError(f"{name}: a matrix on the current GPU is needed")
    n, c = shape
    if (rows is not None and n != rows) or (cols is not None and c != cols):
        raise ValueError(f"{name}: shape {tuple(shape)}, expected ({rows}, {cols})")
    if dtype is not None and t.dtype is not dtype:
        raise ValueError(f"{name}: {t.dtype}, expected {dtype}")
    ld, unit = t.stride()
    if unit != 1 and c > 1:
        raise ValueError(f"{name}: the last dimension needs unit stride")
    if n < 2:
        return c or 1
    if ld < c:
        raise ValueError(f"{name}: rows overlap")
    return ld or 1


def _flat(t: torch.Tensor, name: str, dev: int, numel: int, dtype) -> int:
    """Checks a contiguous array on GPU ``dev``, the current one; its address."""
    if t.dtype is not dtype or t.numel() != numel or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} array of {numel} elements on the current GPU is needed")
    return t.data_ptr()


def _no_grad(name: str) -> None:
    """For an input that requires a gradient, which would be lost silently."""
    if torch.is_grad_enabled():
        raise ValueError(f"{name} requires a gradient, which is not recorded: call under torch.no_grad() or in an "
                         "autograd.Function, and the gradient's own call for the way back")


# ---------------------------------------------------------------- routing
def route(logits, k: int, *, bias=None, score: str = "softmax", normalise: bool = False, scale: float = 1.0, ids=None,
          weights=None, stream=None):
    """(ids int32 [tokens, k], weights float32 [tokens, k]) of the k largest
    logits + bias a row; see ll_moe_route.  A selection bias that belongs to the
    score, not the logit, chooses other experts and takes the scores instead:

        scores = torch.sigmoid(logits.float())
        ids, _ = moe.route(scores, k, bias=bias)
        weights = scores.gather(1, ids.long())     # divided by their sum, scaled

    with ``route_grad(logits, ids, dweights, score="sigmoid", ...)`` on the way
    back."""
    dev = _device()
    ld = _mat(logits, "logits", dev)
    if logits.requires_grad:
        _no_grad("logits")
    t, e = logits.shape
    if ids is None:
        ids = _new(stream, t, k, dtype=torch.int32, device=logits.device)
    if weights is None:
        weights = _new(stream, t, k, dtype=torch.float32, device=logits.device)
    ll.check(_c.ll_moe_route(logits.data_ptr(), ld, t, e, k, _dt(logits),
                             None if bias is None else _flat(bias, "bias", dev, e, torch.float32), lm.SCORES[score],
                             int(normalise), scale, _flat(ids, "ids", dev, t * k, torch.int32),
                             _flat(weights, "weights", dev, t * k, torch.float32), _stream(stream, dev)),
             "ll_moe_route")
    return ids, weights


def route_grad(logits, ids, dweights, *, score: str = "softmax", normalise: bool = False, scale: float = 1.0,
               out=None, stream=None):
    """The logits' gradient from the weights' gradient, for the ids that route returned."""
    dev = _device()
    ld = _mat(logits, "logits", dev)
    t, e = logits.shape
    k = ids.shape[-1]
    if out is None:
        out = _new(stream, t, e, dtype=logits.dtype, device=logits.device)
    ldd = _mat(out, "out", dev, t, e, logits.dtype)
    ll.check(_c.ll_moe_route_grad(logits.data_ptr(), ld, t, e, k, _dt(logits), lm.SCORES[score], int(normalise),
                                  scale, _flat(ids, "ids", dev, t * k, torch.int32),
                                  _flat(dweights, "dweights", dev, t * k, torch.float32), out.data_ptr(), ldd,
                                  _stream(stream, dev)), "ll_moe_route_grad")
    return out


# ---------------------------------------------------------------- dispatch and combine
class Dispatch:
    """Buffers of a dispatch of up to ``tokens`` tokens with ``k`` choices each
    to the experts [first, first + experts): ``offsets`` [experts + 1],
    ``slots`` [tokens * k], ``rows`` [tokens, k] and the sorted rows ``x``
    [tokens * k, features] (``features`` 0: sort only).  After ``dispatch`` of
    fewer tokens the attributes are views of that many."""

    def __init__(self, tokens: int, k: int, experts: int, features: int, dtype=torch.bfloat16, *, first: int = 0,
                 device="cuda"):
        self.capacity, self.k, self.experts, self.first, self.features = tokens, k, experts, first, features
        st, need = lm.ll_moe_dispatch_bytes(tokens, k, experts)
        ll.check(st, "ll_moe_dispatch_bytes")
        n = tokens * k
        self.offsets = torch.zeros(experts + 1, dtype=torch.int32, device=device)
        self._slots = torch.empty(n, dtype=torch.int32, device=device)
        self._rows = torch.empty(n, dtype=torch.int32, device=device)
        self._x = torch.empty(n, features, dtype=dtype, device=device)
        # fewer tokens may be cut into more blocks than the capacity is, but never into more than this
        self._work = torch.empty(max(need, 128 * experts * 4), dtype=torch.uint8, device=device)
        self._view(tokens)

    def _view(self, tokens: int) -> None:
        n = tokens * self.k
        self.tokens = tokens
        self.slots, self.rows, self.x = self._slots[:n], self._rows[:n].view(tokens, self.k), self._x[:n]

    def dispatch(self, ids, x=None, stream=None):
        """Sorts the (token, choice) pairs of ``ids`` [tokens, k] and, given the
        tokens' rows ``x``, copies them in that order; see ll_moe_dispatch."""
        dev = _device()
        t = ids.shape[0]
        if ids.dim() != 2 or ids.shape[1] != self.k or t > self.capacity:
            raise ValueError(f"ids: shape {tuple(ids.shape)}, expected at most ({self.capacity}, {self.k})")
        xp = ldx = 0
        if x is not None:
            ldx = _mat(x, "x", dev, t, self.features, self._x.dtype)
            if x.requires_grad:
                _no_grad("x")
            xp = x.data_ptr()
        if self.offsets.get_device() != dev:
            raise ValueError("the plan's buffers are not on the current GPU")
        ll.check(_c.ll_moe_dispatch(_flat(ids, "ids", dev, t * self.k, torch.int32), t, self.k, self.first,
                                    self.experts, xp, ldx, self.features, _DT[self._x.dtype],
                                    self.offsets.data_ptr(), self._slots.data_ptr(), self._rows.data_ptr(),
                                    self._x.data_ptr() if xp else 0, self.features, self._work.data_ptr(),
                                    self._work.numel(), _stream(stream, dev)), "ll_moe_dispatch")
        if t != self.tokens:
            self._view(t)
        return self

    def grad(self, dx, out=None, stream=None):
        """The gradient of the tokens' rows from that of the sorted rows."""
        return combine(dx, self.rows, out=out, stream=stream)


def combine(y, rows, weights=None, *, residual=None, out=None, stream=None):
    """out[t] = residual[t] + sum_j weights[t, j] * y[rows[t, j]]; see ll_moe_combine."""
    dev = _device()
    ldy = _mat(y, "y", dev)
    if y.requires_grad or (weights is not None and weights.requires_grad):
        _no_grad("y or weights")
    n, h = y.shape
    t, k = rows.shape
    if out is None:
        out = _new(stream, t, h, dtype=y.dtype, device=y.device)
    ldo = _mat(out, "out", dev, t, h, y.dtype)
    rp = ldr = 0
    if residual is not None:
        ldr, rp = _mat(residual, "residual", dev, t, h, y.dtype), residual.data_ptr()
        if residual.requires_grad:
            _no_grad("residual")
    ll.check(_c.ll_moe_combine(y.data_ptr(), ldy, n, _flat(rows, "rows", dev, t * k, torch.int32),
                               None if weights is None else _flat(weights, "weights", dev, t * k, torch.float32), rp,
                               ldr, t, k, h, _dt(y), out.data_ptr(), ldo, _stream(stream, dev)), "ll_moe_combine")
    return out


def combine_grad(dout, y, rows, weights=None, *, dy=None, dweights=None, stream=None):
    """(dy, dweights) of combine; without weights, dweights is computed only
    where its memory is given, and else None.  Rows of dy that no token uses
    are left as they are (zeros in a new one)."""
    dev = _device()
    ldd = _mat(dout, "dout", dev)
    ldy = _mat(y, "y", dev, None, dout.shape[1], dout.dtype)
    n, h = y.shape
    t, k = rows.shape
    if dout.shape[0] != t:
        raise ValueError(f"dout: {dout.shape[0]} rows, expected {t}")
    if dy is None:
        dy = _new(stream, n, h, dtype=y.dtype, device=y.device, make=torch.zeros)
    lddy = _mat(dy, "dy", dev, n, h, y.dtype)
    wp = wg = None
    if weights is not None:
        wp = _flat(weights, "weights", dev, t * k, torch.float32)
        if dweights is None:
            dweights = _new(stream, t, k, dtype=torch.float32, device=y.device)
    if dweights is not None:
        wg = _flat(dweights, "dweights", dev, t * k, torch.float32)
    ll.check(_c.ll_moe_combine_grad(dout.data_ptr(), ldd, y.data_ptr(), ldy, n,
                                    _flat(rows, "rows", dev, t * k, torch.int32), wp, t, k, h, _dt(y), dy.data_ptr(),
                                    lddy, wg, _stream(stream, dev)), "ll_moe_combine_grad")
    return dy, dweights


# ---------------------------------------------------------------- products
def _weight(w, dev: int, name="w"):
    """(groups, out, in, leading dimension, group stride) of a weight [out, in] or [groups, out, in]."""
    if w.dim() == 2:
        ld = _mat(w, name, dev)
        return 1, w.shape[0], w.shape[1], ld, w.shape[0] * ld
    if w.dim() != 3 or w.get_device() != dev:
        raise ValueError(f"{name}: [out, in] or [groups, out, in] on the current GPU is needed")
    g, o, i = w.shape
    gs, ld, unit = w.stride()
    if i > 1 and unit != 1:
        raise ValueError(f"{name}: the last dimension needs unit stride")
    if o < 2:
        ld = i
    if g < 2:
        gs = o * ld
    return g, o, i, ld, gs


def _offsets(offsets, groups: int, dev: int):
    if offsets is None:
        if groups != 1:
            raise ValueError("offsets are needed for more than one group")
        return None
    return _flat(offsets, "offsets", dev, groups + 1, torch.int32)


_needs: dict = {}  # workspace bytes by shape (host arithmetic only)


def _plan(which: int, stream, device, dt, act, groups, rows, in_, out, offsets, ldx, ldw, wstride, ldy, ldz=0, ldr=0):
    """(descriptor, workspace address, its bytes, the workspace)."""
    d = lm.LLLinearDesc(lm.DESC_SIZE, dt, act, groups, rows, in_, out, offsets, ldx, ldw, wstride, ldy, ldz, ldr)
    # what a plan depends on: the shape, whether there are offsets, and how the operands' rows are aligned
    lds = ldx | ldy if which == lm.LL_LINEAR_GRAD_W else ldw | wstride | (ldy if which else ldx)
    key = (which, dt, act, groups, rows, in_, out, offsets is None, lds & 7)
    need = _needs.get(key)
    if need is None:
        st, need = lm.ll_linear_bytes(d, which)
        ll.check(st, "ll_linear_bytes")
        if len(_needs) >= 4096:
            _needs.clear()
        _needs[key] = need
    if not need:
        return d, None, 0, None
    ws = _new(stream, need, dtype=torch.uint8, device=device)
    return d, ws.data_ptr(), need, ws


def linear(x, w, *, bias=None, act: str = "none", residual=None, offsets=None, out=None, z=None, stream=None):
    """act(x w^T + bias) + residual, by groups of rows where ``offsets`` is
    given.  ``z`` [rows, out]: receives the pre-activations.  See ll_linear."""
    dev = _device()
    n = x.shape[0]
    g, o, i, ldw, gs = _weight(w, dev)
    ldx = _mat(x, "x", dev, n, i, w.dtype)
    if x.requires_grad or w.requires_grad or (bias is not None and bias.requires_grad):
        _no_grad("x, w or bias")
    width = o // 2 if act in lm.GATED else o
    if out is None:
        out = _new(stream, n, width, dtype=x.dtype, device=x.device)
    ldy = _mat(out, "out", dev, n, width, x.dtype)
    ldr = ldz = max(o, 1)
    rp = zp = None
    if residual is not None:
        ldr, rp = _mat(residual, "residual", dev, n, width, x.dtype), residual.data_ptr()
        if residual.requires_grad:
            _no_grad("residual")
    if z is not None:
        ldz, zp = _mat(z, "z", dev, n, o, x.dtype), z.data_ptr()
    d, wp, wn, _ws = _plan(lm.LL_LINEAR_FORWARD, stream, x.device, _dt(x), lm.ACTS[act], g, n, i, o,
                           _offsets(offsets, g, dev), ldx, ldw, gs, ldy, ldz, ldr)
    ll.check(_c.ll_linear(d, x.data_ptr(), w.data_ptr(),
                          None if bias is None else _flat(bias, "bias", dev, g * o, x.dtype), rp, out.data_ptr(), zp,
                          wp, wn, _stream(stream, dev)), "ll_linear")
    return out


def linear_grad_x(dz, w, *, act: str = "none", z=None, offsets=None, out=None, stream=None):
    """dz w, taken on through the activation of the layer below whose
    pre-activations are ``z``; see ll_linear_grad_x."""
    dev = _device()
    n = dz.shape[0]
    g, o, i, ldw, gs = _weight(w, dev)
    ldy = _mat(dz, "dz", dev, n, o, w.dtype)
    width = 2 * i if act in lm.GATED else i
    if out is None:
        out = _new(stream, n, width, dtype=dz.dtype, device=dz.device)
    ldx = _mat(out, "out", dev, n, width, dz.dtype)
    ldz, zp = width, None
    if act != "none":
        if z is None:
            raise ValueError("z is needed to go through an activation")
        ldz, zp = _mat(z, "z", dev, n, width, dz.dtype), z.data_ptr()
    d, wp, wn, _ws = _plan(lm.LL_LINEAR_GRAD_X, stream, dz.device, _dt(dz), lm.ACTS[act], g, n, i, o,
                           _offsets(offsets, g, dev), ldx, ldw, gs, ldy, ldz)
    ll.check(_c.ll_linear_grad_x(d, dz.data_ptr(), w.data_ptr(), zp, out.data_ptr(), wp, wn, _stream(stream, dev)),
             "ll_linear_grad_x")
    return out


def linear_grad_w(dz, x, *, offsets=None, out=None, bias_out=None, add: bool = False, stream=None):
    """(dw, dbias): dw [out, in] (or [groups, out, in] with offsets) = dz^T x,
    dbias its bias gradient where ``bias_out`` is given.  Their type is dz's
    or float32; ``add`` adds to what they hold.  See ll_linear_grad_w."""
    dev = _device()
    n, o = dz.shape
    ldy = _mat(dz, "dz", dev)
    ldx = _mat(x, "x", dev, n, None, dz.dtype)
    i = x.shape[1]
    groups = 1 if offsets is None else offsets.numel() - 1
    if out is None:
        shape = (o, i) if offsets is None else (groups, o, i)
        out = _new(stream, *shape, dtype=dz.dtype, device=dz.device, make=torch.zeros if add else torch.empty)
    g, o2, i2, ldw, gs = _weight(out, dev, "out")
    if (g, o2, i2) != (groups, o, i) or out.dtype not in (dz.dtype, torch.float32):
        raise ValueError(f"out: {tuple(out.shape)} {out.dtype}, expected ({groups}, {o}, {i})")
    flags = (lm.LL_GRAD_F32 if out.dtype == torch.float32 else 0) | (lm.LL_GRAD_ADD if add else 0)
    bp = None if bias_out is None else _flat(bias_out, "bias_out", dev, g * o, out.dtype)
    d, wp, wn, _ws = _plan(lm.LL_LINEAR_GRAD_W, stream, dz.device, _dt(dz), lm.LL_ACT_NONE, g, n, i, o,
                           _offsets(offsets, g, dev), ldx, ldw, gs, ldy)
    ll.check(_c.ll_linear_grad_w(d, dz.data_ptr(), x.data_ptr(), out.data_ptr(), bp, flags, wp, wn,
                                 _stream(stream, dev)), "ll_linear_grad_w")
    return out, bias_out


def act_grad(dy, z, act: str, *, out=None, stream=None):
    """The gradient of an activation's output taken to its pre-activations z."""
    dev = _device()
    ldy = _mat(dy, "dy", dev)
    n, h = dy.shape
    width = 2 * h if act in lm.GATED else h
    ldz = _mat(z, "z", dev, n, width, dy.dtype)
    if out is None:
        out = _new(stream, n, width, dtype=dy.dtype, device=dy.device)
    ldo = _mat(out, "out", dev, n, width, dy.dtype)
    ll.check(_c.ll_act_grad(dy.data_ptr(), ldy, z.data_ptr(), ldz, n, h, _dt(dy), lm.ACTS[act], out.data_ptr(), ldo,
                            _stream(stream, dev)), "ll_act_grad")
    return out


# ---------------------------------------------------------------- 8 bits
def scales_of(*shape, device="cuda", stream=None) -> torch.Tensor:
    """Memory for scales of ``shape`` (the last is the number of blocks a row):
    a row starts at a multiple of 4 bytes, which is what the calls below need."""
    wide = _new(stream, *shape[:-1], (shape[-1] + 3) // 4 * 4, dtype=torch.uint8, device=device)
    return wide.view(E8M0)[..., :shape[-1]]


def _codes_for(stream, *shape, device) -> torch.Tensor:
    """Memory for codes, whose rows start at multiples of 16 bytes: products load
    those straight into shared memory."""
    wide = (shape[-1] + 15) // 16 * 16
    t = _new(stream, *shape[:-1], wide, dtype=E4M3, device=device)
    return t if wide == shape[-1] else t[..., :shape[-1]]


def _like(t, name: str, dev: int, rows: int, cols: int, dtype) -> int:
    """_mat, sooner done where the rows are contiguous."""
    if t.shape == (rows, cols) and t.dtype is dtype and t.is_contiguous() and t.get_device() == dev:
        return cols or 1
    return _mat(t, name, dev, rows, cols, dtype)


def _codes(t, name: str, dev: int, rows: int, cols: int) -> int:
    return _like(t, name, dev, rows, cols, E4M3)


def _scale_rows(t, name: str, dev: int, rows: int, blocks: int) -> int:
    """Checks a matrix of scales; its leading dimension."""
    if t.dtype is not E8M0 or t.shape != (rows, blocks) or t.get_device() != dev:
        raise ValueError(f"{name}: {tuple(t.shape)} {t.dtype}, expected ({rows}, {blocks}) {E8M0} on the current GPU")
    ld, unit = t.stride()
    wide = (blocks + 3) // 4 * 4
    if (blocks > 1 and unit != 1) or (rows > 1 and (ld % 4 or ld < blocks)) or t.data_ptr() % 4:
        raise ValueError(f"{name}: rows of scales start at multiples of 4 bytes (moe.scales_of makes such memory)")
    if rows < 2:
        ld = wide
    if wide != blocks:
        _readable(t, name, (rows - 1) * ld + wide)
    return ld


def _readable(t, name: str, nbytes: int) -> None:
    """Scales are read four at a time: the last row's four have to be there."""
    if t.numel() and t.untyped_storage().nbytes() - t.storage_offset() < nbytes:
        raise ValueError(f"{name}: the last row's memory ends inside four scales (moe.scales_of makes longer rows)")


def quantise(x, *, act: str = "none", offsets=None, out=None, scales=None, stream=None):
    """(out, scales): act(x) in 8 bits (float8_e4m3fn [rows, features]) with a
    power of two (float8_e8m0fnu [rows, ceil(features / 128)]) for each 128
    features of a row; see ll_quantise.  Memory it makes has rows at multiples of
    16 codes and of 4 scales.  With ``offsets``, rows behind the last
    group are left as they are."""
    dev = _device()
    ldx = _mat(x, "x", dev)
    if x.requires_grad:
        _no_grad("x")
    n, width = x.shape
    if act in lm.GATED and width % 2:
        raise ValueError(f"x: {width} features, a gated activation needs an even number")
    h = width // 2 if act in lm.GATED else width
    if out is None:
        out = _codes_for(stream, n, h, device=x.device)
    if scales is None:
        scales = scales_of(n, (h + 127) // 128, device=x.device, stream=stream)
    end = None
    if offsets is not None:
        if offsets.numel() == 0:
            raise ValueError("offsets: none")
        end = _flat(offsets, "offsets", dev, offsets.numel(), torch.int32) + (offsets.numel() - 1) * 4
    ldq, lds = _codes(out, "out", dev, n, h), _scale_rows(scales, "scales", dev, n, (h + 127) // 128)
    ll.check(_c.ll_quantise(x.data_ptr(), ldx, n, end, h, _dt(x), lm.ACTS[act], out.data_ptr(), ldq,
                            scales.data_ptr(), lds, _stream(stream, dev)), "ll_quantise")
    return out, scales


def _weight_scales(t, name: str, dev: int, groups: int, rows: int, blocks: int):
    """(leading dimension, group stride) of scales [rows, blocks] or [groups, rows, blocks]."""
    if t.dim() == 2 and groups == 1:
        return _scale_rows(t, name, dev, rows, blocks), 0
    if t.dim() != 3 or t.shape[0] != groups:
        raise ValueError(f"{name}: {tuple(t.shape)}, expected ({groups}, {rows}, {blocks})")
    ld = _scale_rows(t[0], name, dev, rows, blocks)
    stride = t.stride(0) if groups > 1 else 0
    if stride % 4:
        raise ValueError(f"{name}: groups of scales start at multiples of 4 bytes")
    _readable(t, name, (groups - 1) * stride + (rows - 1) * ld + (blocks + 3) // 4 * 4)
    return ld, stride


def quantise_weight(w, *, transpose: bool = False, out=None, scales=None, stream=None):
    """(out, scales): a weight [out, in] or [groups, out, in] in 8 bits with a
    power of two for each 128 x 128 of it; ``transpose``: as [.., in, out], for
    the gradient of the product's input.  See ll_quantise_weight."""
    dev = _device()
    g, o, i, ldw, gs = _weight(w, dev)
    if w.requires_grad:
        _no_grad("w")
    rows, cols = (i, o) if transpose else (o, i)
    lead = () if w.dim() == 2 else (g,)
    if out is None:
        out = _codes_for(stream, *lead, rows, cols, device=w.device)
    if scales is None:
        scales = scales_of(*lead, (rows + 127) // 128, (cols + 127) // 128, device=w.device, stream=stream)
    if out.dtype is not E4M3 or out.dim() != w.dim():
        raise ValueError(f"out: {tuple(out.shape)} {out.dtype}, expected {(*lead, rows, cols)} {E4M3}")
    g2, r2, c2, ldq, qs = _weight(out, dev, "out")
    if (g2, r2, c2) != (g, rows, cols):
        raise ValueError(f"out: {tuple(out.shape)}, expected {(*lead, rows, cols)}")
    lds, ss = _weight_scales(scales, "scales", dev, g, (rows + 127) // 128, (cols + 127) // 128)
    ll.check(_c.ll_quantise_weight(w.data_ptr(), ldw, gs, g, o, i, _dt(w), int(transpose), out.data_ptr(), ldq, qs,
                                   scales.data_ptr(), lds, ss, _stream(stream, dev)), "ll_quantise_weight")
    return out, scales


def linear8(x, x_scales, w, w_scales, *, bias=None, act: str = "none", residual=None, offsets=None, dtype=None,
            out=None, z=None, stream=None):
    """``linear`` of rows and weights in 8 bits (``quantise``,
    ``quantise_weight``): act(x w^T + bias) + residual, by groups of rows where
    ``offsets`` is given.  bias, residual, z and the result are of type
    ``dtype`` (bfloat16 unless ``out`` or this says otherwise).  See ll_linear8.

    For bfloat16 results products are cut off 2^-13 below the largest of eight
    consecutive ones, about 2^-15 of a result of normal values (they are rounded at
    2^-9): more where a sum's terms cancel than its rounding loses.  With
    dtype=torch.float32 products and sums are binary32.

    The gradient of x is ``linear8`` of the rows' gradient and the transposed
    weight, both in 8 bits, then ``act_grad`` through an activation below; the
    weight's is ``linear_grad_w`` on the rows as they were before."""
    dev = _device()
    n = x.shape[0]
    if w.dtype is not E4M3:
        raise ValueError(f"w: {w.dtype}, expected {E4M3}")
    g, o, i, ldw, gs = _weight(w, dev)
    ldx = _codes(x, "x", dev, n, i)
    kb = (i + 127) // 128
    ldxs = _scale_rows(x_scales, "x_scales", dev, n, kb)
    ldws, ss = _weight_scales(w_scales, "w_scales", dev, g, (o + 127) // 128, kb)
    if (bias is not None and bias.requires_grad) or (residual is not None and residual.requires_grad):
        _no_grad("bias or residual")
    width = o // 2 if act in lm.GATED else o
    if dtype is None:
        dtype = torch.bfloat16 if out is None else out.dtype
    if out is None:
        out = _new(stream, n, width, dtype=dtype, device=x.device)
    ldy = _like(out, "out", dev, n, width, dtype)
    ldr = ldz = max(o, 1)
    rp = zp = None
    if residual is not None:
        ldr, rp = _like(residual, "residual", dev, n, width, dtype), residual.data_ptr()
    if z is not None:
        ldz, zp = _like(z, "z", dev, n, o, dtype), z.data_ptr()
    d = lm.LLLinearDesc(lm.DESC_SIZE, _dt(out), lm.ACTS[act], g, n, i, o, _offsets(offsets, g, dev), ldx, ldw, gs, ldy,
                        ldz, ldr)
    key = (d.dt, d.act, g, n, i, o, offsets is None, ldx & 15, ldw & 15, gs & 15)
    need = _needs8.get(key)
    if need is None:
        st, need = lb.ll_linear8_bytes(d)
        ll.check(st, "ll_linear8_bytes")
        if len(_needs8) >= 4096:
            _needs8.clear()
        _needs8[key] = need
    ws = _new(stream, need, dtype=torch.uint8, device=x.device) if need else None
    ll.check(_c.ll_linear8(d, x.data_ptr(), x_scales.data_ptr(), ldxs, w.data_ptr(), w_scales.data_ptr(), ldws, ss,
                           None if bias is None else _flat(bias, "bias", dev, g * o, dtype), rp, out.data_ptr(), zp,
                           None if ws is None else ws.data_ptr(), need, _stream(stream, dev)), "ll_linear8")
    return out


_needs8: dict = {}  # workspace bytes by shape (host arithmetic only)


# ---------------------------------------------------------------- norms around a block
class Normed(NamedTuple):
    h: Optional[torch.Tensor]         # the next block's input
    r: Optional[torch.Tensor]         # the residual stream
    q: Optional[torch.Tensor]         # h in 8 bits
    q_scales: Optional[torch.Tensor]


class NormGrads(NamedTuple):
    dr: torch.Tensor                  # of the residual stream before and behind the block's output was added
    dy: Optional[torch.Tensor]
    dgate: Optional[torch.Tensor]
    dweight: Optional[torch.Tensor]
    dpost: Optional[torch.Tensor]


def _norm_weights(post, weight, rows, dev: int):
    """(their type's code, addresses) of a norm's weights."""
    kind = weight.dtype if weight is not None else post.dtype if post is not None else torch.float32
    if kind is not rows.dtype and kind is not torch.float32:
        raise ValueError(f"weight or post: {kind}, expected {rows.dtype} or float32")
    f = rows.shape[1]
    pp = None if post is None else _flat(post, "post", dev, f, kind)
    return _DT.get(kind, ll.LL_F32), (pp, None if weight is None else _flat(weight, "weight", dev, f, kind))


def norm(y, weight=None, *, residual=None, gate=None, scale: float = 1.0, post=None, eps: float = 1e-6,
         quantised: bool = False, h=None, r=None, q=None, q_scales=None, stream=None) -> Normed:
    """What stands between two blocks, in one pass (see ll_norm):

        u = post * y / sqrt(mean(y^2) + eps)        the block's own norm (without post: u = y)
        r = residual + scale * gate * u             gate: float32, one a token
        h = weight * r / sqrt(mean(r^2) + eps)      the next block's input (without weight: none)

    ``norm(y, weight).h`` is a plain norm of y; r is computed where anything is
    done to y, or where its memory is given.  ``quantised`` (or q given): h in 8
    bits too, as ``quantise`` makes it.  r may be the residual's own memory."""
    dev = _device()
    ldy = _mat(y, "y", dev)
    n, f = y.shape
    dt, device = y.dtype, y.device
    if torch.is_grad_enabled():
        for t, name in ((y, "y"), (residual, "residual"), (gate, "gate"), (post, "post"), (weight, "weight")):
            if t is not None and t.requires_grad:
                _no_grad(name)
    wdt, (pp, wp) = _norm_weights(post, weight, y, dev)
    if weight is None and (quantised or q is not None or h is not None):
        raise ValueError("weight is needed for h")
    if r is None and (weight is None or residual is not None or gate is not None or post is not None or scale != 1):
        r = _new(stream, n, f, dtype=dt, device=device)
    if h is None and weight is not None:
        h = _new(stream, n, f, dtype=dt, device=device)
    if q is None and quantised:
        q = _codes_for(stream, n, f, device=device)
    xp = gp = rp = hp = qp = sp = None
    ldx = ldr = ldh = ldq = f
    lds = 0
    if residual is not None:
        ldx, xp = _like(residual, "residual", dev, n, f, dt), residual.data_ptr()
    if gate is not None:
        gp = _flat(gate, "gate", dev, n, torch.float32)
    if r is not None:
        ldr, rp = _like(r, "r", dev, n, f, dt), r.data_ptr()
    if h is not None:
        ldh, hp = _like(h, "h", dev, n, f, dt), h.data_ptr()
    if q is not None:
        if q_scales is None:
            q_scales = scales_of(n, (f + 127) // 128, device=device, stream=stream)
        ldq, lds = _codes(q, "q", dev, n, f), _scale_rows(q_scales, "q_scales", dev, n, (f + 127) // 128)
        qp, sp = q.data_ptr(), q_scales.data_ptr()
    d = _norm_desc(_dt(y), wdt, eps, scale, n, f, ldy, ldx, ldr, ldh, ldq, lds, f, f, f)
    ll.check(_c.ll_norm(d, y.data_ptr(), xp, gp, pp, wp, rp, hp, qp, sp, _stream(stream, dev)), "ll_norm")
    return Normed(h, r, q, None if q is None else q_scales)


_norm_descs: dict = {}  # by their own fields: a descriptor is only read
_norm_needs: dict = {}  # workspace bytes by rows and features


def _norm_desc(*fields):
    d = _norm_descs.get(fields)
    if d is None:
        if len(_norm_descs) >= 4096:
            _norm_descs.clear()
        d = _norm_descs[fields] = lb.LLNormDesc(lb.NORM_DESC_SIZE, *fields)
    return d


def norm_grad(dh, r, weight=None, *, dr=None, y=None, gate=None, scale: float = 1.0, post=None, eps: float = 1e-6,
              dr_out=None, dy=None, dgate=None, dweight=None, dpost=None, add: bool = False, stream=None) -> NormGrads:
    """The gradients of ``norm`` from those of h (``dh``) and of r (``dr``), for
    the r it returned (y itself where it returned none); see ll_norm_grad.  dr
    of the result is the residual's gradient.  dy is computed where the block's
    output was normed, gated or scaled, or where its memory is given (else it is
    the result's dr); dgate and dpost where there is a gate and a post, dweight
    (and dpost) in float32, ``add``: added to what their memory holds.  Without
    ``weight``, dh and r are None."""
    dev = _device()
    rows = dr if weight is None else dh
    if rows is None or (weight is None and dh is not None):
        raise ValueError("dh goes with weight; without, dr is needed")
    ld = _mat(rows, "dr" if weight is None else "dh", dev)
    n, f = rows.shape
    dt = rows.dtype
    wdt, (pp, wp) = _norm_weights(post, weight, rows, dev)
    if y is None and (post is not None or gate is not None):
        raise ValueError("y is needed for the gradients of a gate and of the block's own norm")
    if add and ((weight is not None and dweight is None) or (post is not None and dpost is None)):
        raise ValueError("add needs the memory that is added to")

    def fresh(*shape, dtype=dt):
        return _new(stream, *shape, dtype=dtype, device=rows.device)

    changed = post is not None or gate is not None or scale != 1
    if dr_out is None:
        dr_out = fresh(n, f)
    if dy is None and changed:
        dy = fresh(n, f)
    if gate is not None and dgate is None:
        dgate = fresh(n, dtype=torch.float32)
    if weight is not None and dweight is None:
        dweight = fresh(f, dtype=torch.float32)
    if post is not None and dpost is None:
        dpost = fresh(f, dtype=torch.float32)

    def mat(t, name):
        return f if t is None else _like(t, name, dev, n, f, dt)

    def flat(t, name, numel):
        return None if t is None else _flat(t, name, dev, numel, torch.float32)

    def at(t):
        return None if t is None else t.data_ptr()

    d = _norm_desc(_dt(rows), wdt, eps, scale, n, f, mat(y, "y"), f, mat(r, "r"), f if weight is None else ld, f, 0,
                   mat(dr, "dr"), mat(dr_out, "dr_out"), mat(dy, "dy"))
    ws, need = None, 0
    if dweight is not None or dpost is not None:
        need = _norm_needs.get((n, f))
        if need is None:
            st, need = lb.ll_norm_bytes(d)
            ll.check(st, "ll_norm_bytes")
            if len(_norm_needs) >= 4096:
                _norm_needs.clear()
            _norm_needs[n, f] = need
        ws = _new(stream, need, dtype=torch.uint8, device=rows.device)
    ll.check(_c.ll_norm_grad(d, at(dh), at(r) if weight is not None else None, at(dr), at(y), flat(gate, "gate", n), pp,
                             wp, at(dr_out), at(dy), flat(dgate, "dgate", n), flat(dweight, "dweight", f),
                             flat(dpost, "dpost", f), lm.LL_GRAD_ADD if add else 0, at(ws), need,
                             _stream(stream, dev)), "ll_norm_grad")
    return NormGrads(dr_out, dy if dy is not None else dr_out, dgate, dweight, dpost)
