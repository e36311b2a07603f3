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

import torch

from . import llcoll as ll
from . import llmoe as lm

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
