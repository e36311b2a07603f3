"""A weight update on torch tensors (``ll_adamw`` of ``include/llblock.h``).

    opt = AdamW(params, lr=3e-4, weight_decay=0.1, states="8bit", floor=True)
    opt.step(grads)

A step is one small launch and one for each 40 tensors, on the current stream
(or ``stream``).  It counts in device memory, so that a step captured into a
graph is the next one each time the graph is replayed.
"""
from __future__ import annotations

import contextlib
import ctypes
import warnings
from operator import attrgetter
from typing import Optional, Sequence

import numpy as np
import torch
from torch.autograd.graph import increment_version

from . import llblock as lb
from . import llcoll as ll
from .moe import _device, _flat, _stream

_DT = {torch.float32: ll.LL_F32, torch.bfloat16: ll.LL_BF16}
STATES = {"f32": 32, "8bit": 8}
_TYPES = {32: (torch.float32, torch.float32), 8: (torch.float8_e4m3fn, torch.float8_e5m2)}

# of a list of tensors, by map: less host work than a comprehension
_dtype, _numel, _ptr = attrgetter("dtype"), torch.Tensor.numel, torch.Tensor.data_ptr
_contiguous, _get_device = torch.Tensor.is_contiguous, torch.Tensor.get_device

# what changes from step to step of a row of ll_adamw's table
_ROW = np.dtype({"names": ["param", "grad", "gdt"], "formats": [np.uint64, np.uint64, np.int32],
                 "offsets": [getattr(lb.LLAdamwTensor, f).offset for f in ("param", "grad", "gdt")], "itemsize": ctypes.sizeof(lb.LLAdamwTensor)})


class AdamW:
    """Adam with decoupled weight decay over ``params`` (contiguous float32 or
    bfloat16 tensors of one GPU, which are updated in place); see ll_adamw.

    A bfloat16 parameter has a float32 master, made from it, which holds its value:
    a step writes the parameter from it, whatever is there and wherever its memory is
    by then.  Call ``read_params`` where a parameter has got other values than a step's,
    in its memory or with another one.  The states of all
    parameters lie in one tensor each, a parameter's at a multiple of 128
    (``offsets``): ``m`` and ``v`` in float32, or with states="8bit" m as
    float8_e4m3fn and v as float8_e5m2 with a power of two (float8_e8m0fnu) for
    each 128 values.  States in 8 bits are rounded at random, by ``seed``; with
    ``floor`` a v above 0 is never rounded to 0 (LL_ADAMW_FLOOR).  Without it a value
    whose gradients are 2^-14 and less of the largest of its 128 can move by a thousand
    times lr in a step; floor=False is for runs that have to go on as they were.
    Values between a parameter's last and the next multiple of 128 stay 0.

    ``state``: a ``state_dict()`` to go on from, whose tensors are used, not
    copied.  The options may be changed between steps (``opt.lr = ...``).  Steps of
    one optimiser follow one another: two at once, on two streams, are not
    meant.  Its memory is of the stream it was made on: keep it until steps on
    other streams have run."""

    def __init__(self, params: Sequence[torch.Tensor], *, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8,
                 weight_decay: float = 0.0, states: str = "f32", seed: int = 0, state: Optional[dict] = None,
                 floor: Optional[bool] = None):
        self.params = list(params)
        self.lr, self.betas, self.eps, self.weight_decay = lr, tuple(betas), eps, weight_decay
        self.seed = seed
        if states not in STATES:
            raise ValueError(f"states: {states!r}, expected one of {sorted(STATES)}")
        self.bits = STATES[states]
        if self.bits == 8 and floor is None:
            warnings.warn("8-bit states without floor=True: values whose gradients are far below the largest of their 128 can "
                          "move by many times lr (floor=False says that this is meant)", stacklevel=2)
        if not self.params:
            raise ValueError("params: none")
        dev = self.params[0].get_device()
        self._dev = dev
        self.offsets, total = [], 0
        for i, p in enumerate(self.params):
            if p.dtype not in _DT:
                raise ll.LLError(ll.LL_ERR_UNSUPPORTED, str(p.dtype))
            if dev < 0 or p.get_device() != dev or not p.is_contiguous():
                raise ValueError(f"params[{i}]: a contiguous tensor is needed, all on one GPU")
            self.offsets.append(total)
            total += (p.numel() + 127) // 128 * 128
        self._apart()
        device = self.params[0].device
        mt, vt = _TYPES[self.bits]
        eight = self.bits == 8
        if state is None:
            state = {"masters": [p.detach().float() if p.dtype is torch.bfloat16 else None for p in self.params],
                     "m": torch.zeros(total, dtype=torch.uint8, device=device).view(mt) if eight
                     else torch.zeros(total, dtype=mt, device=device),
                     "v": torch.zeros(total, dtype=torch.uint8, device=device).view(vt) if eight
                     else torch.zeros(total, dtype=vt, device=device),
                     "m_scales": _ones(total // 128, device) if eight else None,
                     "v_scales": _ones(total // 128, device) if eight else None,
                     "count": torch.zeros(1, dtype=torch.int32, device=device)}
        self._check_state(state, total, mt, vt)
        self.masters, self.m, self.v = state["masters"], state["m"], state["v"]
        self.m_scales, self.v_scales, self.count = state["m_scales"], state["v_scales"], state["count"]
        self.floor = bool(floor)
        self._work = torch.empty(lb.LL_ADAMW_WORKSPACE, dtype=torch.uint8, device=device)
        self._table = (lb.LLAdamwTensor * len(self.params))()
        self._fields = np.frombuffer(self._table, dtype=_ROW)  # the same memory
        self._sizes, self._dtypes = [p.numel() for p in self.params], [p.dtype for p in self.params]
        self._fields["param"] = self._at = list(map(_ptr, self.params))
        self._grad_dtypes: list = []  # the gradients' types there
        self._versioned = [p for p in self.params if not p.is_inference()]
        es = 1 if eight else 4
        for t, p, w, at in zip(self._table, self.params, self.masters, self.offsets):
            t.n, t.at, t.dt = p.numel(), at, _DT[p.dtype]
            t.master = None if w is None else w.data_ptr()
            t.m, t.v = self.m.data_ptr() + at * es, self.v.data_ptr() + at * es
            if eight:
                t.m_scales, t.v_scales = self.m_scales.data_ptr() + at // 128, self.v_scales.data_ptr() + at // 128

    def _check(self, grads, dev: int) -> None:
        """One contiguous tensor of a parameter's size and a known type each; their types go into the table."""
        if list(map(_numel, grads)) != self._sizes or list(map(_get_device, grads)) != [dev] * len(self._sizes) \
                or not all(map(_contiguous, grads)):
            raise ValueError("grads: one contiguous tensor on the parameters' GPU a parameter, of its number of values, "
                             "is needed")
        types = list(map(_dtype, grads))
        if types != self._grad_dtypes:
            try:
                self._fields["gdt"] = [_DT[t] for t in types]
            except KeyError as e:
                raise ll.LLError(ll.LL_ERR_UNSUPPORTED, str(e)) from None
            self._grad_dtypes = types

    def _apart(self) -> None:
        """Two parameters in the same memory would be updated at the same time."""
        spans = sorted((p.data_ptr(), p.numel() * p.element_size(), i) for i, p in enumerate(self.params) if p.numel())
        for (at, size, _), (behind, _, i) in zip(spans, spans[1:]):
            if behind < at + size:
                raise ValueError(f"params[{i}]: given twice, or shares memory with another")

    def _check_state(self, state: dict, total: int, mt, vt) -> None:
        dev = self._dev
        if len(state["masters"]) != len(self.params):
            raise ValueError(f"masters: {len(state['masters'])}, expected {len(self.params)}")
        for i, (p, w) in enumerate(zip(self.params, state["masters"])):
            if (w is None) != (p.dtype is torch.float32):
                raise ValueError(f"masters[{i}]: one goes with a bfloat16 parameter")
            if w is not None:
                _flat(w, f"masters[{i}]", dev, p.numel(), torch.float32)
        _flat(state["m"], "m", dev, total, mt)
        _flat(state["v"], "v", dev, total, vt)
        _flat(state["count"], "count", dev, 1, torch.int32)
        for name in ("m_scales", "v_scales"):
            if self.bits == 8:
                _flat(state[name], name, dev, total // 128, torch.float8_e8m0fnu)
            elif state[name] is not None:
                raise ValueError(f"{name}: states in float32 have none")

    @property
    def floor(self) -> bool:
        return self._floor

    @floor.setter
    def floor(self, on: bool) -> None:
        """On states that were made without it, a v of 0 beside an m goes up to its least code."""
        self._floor = bool(on)
        if on and self.bits == 8:
            m, v = self.m.view(torch.uint8), self.v.view(torch.uint8)
            v.masked_fill_((v == 0) & ((m & 0x7F) != 0), 1)

    def state_dict(self) -> dict:
        """The state's own tensors (``AdamW(..., state=...)`` goes on from them)."""
        return {"masters": self.masters, "m": self.m, "v": self.v, "m_scales": self.m_scales,
                "v_scales": self.v_scales, "count": self.count}

    def read_params(self, stream=None) -> None:
        """Takes up what the bfloat16 parameters hold now: a value that is not its master
        rounded becomes its master.  The others keep the bits that a parameter does not
        have."""
        with torch.no_grad(), contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):
            for p, w in zip(self.params, self.masters):
                if w is not None:
                    p, w = p.detach().reshape(-1), w.view(-1)
                    w.copy_(torch.where(w.to(p.dtype) == p, w, p.float()))

    def step(self, grads: Sequence[torch.Tensor], *, lr=None, grad_scale=None, stream=None) -> None:
        """One update.  ``grads``: one contiguous float32 or bfloat16 tensor a
        parameter.  ``lr``: this step's, a number or a float32 tensor of one
        value; ``grad_scale``: a float32 tensor of one value that gradients are
        multiplied by.  Tensors are read when the step runs, so a captured step
        takes what they hold then."""
        dev = _device()
        if dev != self._dev:
            raise ValueError("the parameters are not on the current GPU")
        table, fields = self._table, self._fields
        self._check(grads, dev)
        fields["grad"] = list(map(_ptr, grads))
        # (other memory may lie at the same address, or the same memory be strided otherwise)
        if list(map(_numel, self.params)) != self._sizes or list(map(_dtype, self.params)) != self._dtypes \
                or not all(map(_contiguous, self.params)):
            raise ValueError("params: their sizes, types or strides have changed")
        at = list(map(_ptr, self.params))
        if at != self._at:  # a parameter's memory is another than at the last step
            if list(map(_get_device, self.params)) != [dev] * len(at):
                raise ValueError("params: not all on the GPU they were on")
            self._apart()
            fields["param"] = self._at = at
        rate, rate_at = self.lr if lr is None else lr, None
        if isinstance(rate, torch.Tensor):
            rate, rate_at = 0.0, _flat(rate, "lr", dev, 1, torch.float32)
        bits = self.bits | (lb.LL_ADAMW_FLOOR if self.floor and self.bits == 8 else 0)
        d = lb.LLAdamwDesc(lb.ADAMW_DESC_SIZE, bits, rate, self.betas[0], self.betas[1], self.eps,
                           self.weight_decay, self.seed & 0xFFFFFFFF)
        ll.check(lb.ll_adamw(d, table, len(table), self.count.data_ptr(), rate_at,
                             None if grad_scale is None else _flat(grad_scale, "grad_scale", dev, 1, torch.float32),
                             self._work.data_ptr(), lb.LL_ADAMW_WORKSPACE, _stream(stream, dev)), "ll_adamw")
        increment_version(self._versioned)  # a backward pass that still needs the old values says so


def _ones(n: int, device) -> torch.Tensor:
    """Scales of 1."""
    return torch.full((n,), 127, dtype=torch.uint8, device=device).view(torch.float8_e8m0fnu)
