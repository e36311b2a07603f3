"""A mixture-of-experts layer over the virtual ranks: the expert-layer operators
(``moe``) between the collectives they stand next to in an expert-parallel
program.

Rank r holds ``tokens`` of the batch and experts [r * E / P, (r + 1) * E / P);
the router's weight is on every rank.  The router runs in binary32 whatever the
layer's type: logits rounded to bfloat16 would tie, and choose other experts.
Forward, on each rank:

    x    = AllGather of the ranks' tokens
    ids, weights = route(x w_router^T)
    y    = down(silu(gate) * up) of the rows dispatched to this rank's experts
    part = combine(y, weights), straight into the rank's slice
    out  = ReduceScatter of part

Backward runs the same two collectives the other way round: AllGather of the
outputs' gradient, the operators' gradients, ReduceScatter of the inputs'
gradient, and an AllReduce of the router's.

With products="e4m3" the experts' two products and the gradients of their rows
run in 8 bits: rows are quantised as they come, weights once for all steps
between two updates; the weights' gradients and the router keep their types.

``ExpertBlock`` is the layer between two norms, on a residual stream, with its
weight update.

One process drives all the ranks here, so what a rank computes is a loop over
ranks; every step of it uses that rank's own buffers only.

    python -m paper_2607_16100_amd.expert_layer      # training steps, timed
"""
from __future__ import annotations

import torch

from . import llcoll as ll
from . import moe
from .optim import AdamW
from .region import SymRegion

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


class ExpertLayer:
    """``tokens``: per rank.  Weights are random, scaled by the square root of
    the fan-in; assign ``router`` [E, H] (binary32), ``up`` [P][E/P, 2F, H] and
    ``down`` [P][E/P, H, F] to use others.  ``products``: "same" (as ``dtype``)
    or "e4m3"; then call ``quantise_weights()`` after a change of ``up`` or
    ``down``."""

    def __init__(self, nranks: int, tokens: int, hidden: int, ffn: int, experts: int, k: int, dtype: str = "bf16",
                 seed: int = 0, device="cuda", products: str = "same"):
        if experts % nranks:
            raise ValueError(f"{experts} experts over {nranks} ranks")
        if products not in ("same", "e4m3"):
            raise ValueError(f"products: {products!r}, expected 'same' or 'e4m3'")
        self.nranks, self.tokens, self.hidden, self.k = nranks, tokens, hidden, k
        self.local = experts // nranks
        self.dtype = _TORCH[dtype]
        n = nranks * tokens
        self._gather = SymRegion(nranks, tokens * hidden, dtype, out_elems=nranks * n * hidden)
        self._scatter = SymRegion(nranks, n * hidden, dtype, out_elems=n * hidden)
        self._sum = SymRegion(nranks, experts * hidden, "f32", out_elems=nranks * experts * hidden)
        for region in (self._gather, self._scatter, self._sum):
            region.init()
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(*shape, dtype=self.dtype):
            return (torch.randn(*shape, generator=g, device=device) * shape[-1] ** -0.5).to(dtype)

        self.router = weight(experts, hidden, dtype=torch.float32)
        self.up = [weight(self.local, 2 * ffn, hidden) for _ in range(nranks)]
        self.down = [weight(self.local, hidden, ffn) for _ in range(nranks)]
        self.plans = [moe.Dispatch(n, k, self.local, hidden, self.dtype, first=r * self.local, device=device)
                      for r in range(nranks)]
        rows = n * k  # as many as a rank can get
        self._z = [torch.empty(rows, 2 * ffn, dtype=self.dtype, device=device) for _ in range(nranks)]
        self._h = [torch.empty(rows, ffn, dtype=self.dtype, device=device) for _ in range(nranks)]
        self._y = [torch.empty(rows, hidden, dtype=self.dtype, device=device) for _ in range(nranks)]
        self._saved = [None] * nranks
        self.products = products
        self._up8 = self._down8 = None
        if products == "e4m3":
            self.quantise_weights()

    def quantise_weights(self, stream=None) -> None:
        """Codes and scales of ``up`` and ``down`` as they are now, and of their
        transposes for the way back; on ``stream``, behind what changed them."""
        if self.products != "e4m3":
            return
        if self._up8 is None:
            self._up8, self._down8 = ([(moe.quantise_weight(w, stream=stream),
                                        moe.quantise_weight(w, transpose=True, stream=stream)) for w in ws]
                                      for ws in (self.up, self.down))
            return
        for held, ws in ((self._up8, self.up), (self._down8, self.down)):
            for ((q, s), (qt, st)), w in zip(held, ws):
                moe.quantise_weight(w, out=q, scales=s, stream=stream)
                moe.quantise_weight(w, transpose=True, out=qt, scales=st, stream=stream)

    # -- the regions as matrices
    def _slice(self, region: SymRegion, r: int, rows: int, cols: int) -> torch.Tensor:
        """Rank r's input area."""
        nbytes = rows * cols * region.esize
        return region.sym.view(self.nranks, -1)[r, :nbytes].view(_TORCH[region.dtype]).view(rows, cols)

    def _out(self, region: SymRegion, r: int, rows: int, cols: int) -> torch.Tensor:
        """Rank r's output."""
        nbytes = rows * cols * region.esize
        return region.out[r * nbytes:(r + 1) * nbytes].view(_TORCH[region.dtype]).view(rows, cols)

    def _all_gather(self, shards: torch.Tensor) -> list:
        if shards.requires_grad:
            moe._no_grad("the layer's input")
        for r in range(self.nranks):
            self._slice(self._gather, r, self.tokens, self.hidden).copy_(shards[r])
        ll.check(self._gather.allgather(self.tokens * self.hidden), "ll_allgather")
        return [self._out(self._gather, r, self.nranks * self.tokens, self.hidden) for r in range(self.nranks)]

    def _reduce_scatter(self) -> torch.Tensor:
        ll.check(self._scatter.reduce_scatter(self.tokens * self.hidden), "ll_reduce_scatter")
        return self._out(self._scatter, 0, self.nranks * self.tokens, self.hidden).view(
            self.nranks, self.tokens, self.hidden).clone()

    # -- passes
    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """[P, tokens, hidden] -> the same shape."""
        n = self.nranks * self.tokens
        for r, xs in enumerate(self._all_gather(x)):
            logits = moe.linear(xs.float(), self.router.float())
            ids, weights = moe.route(logits, self.k, normalise=True)
            plan = self.plans[r].dispatch(ids, xs)
            off = plan.offsets
            if self.products == "e4m3":
                moe.linear8(*moe.quantise(plan.x, offsets=off), *self._up8[r][0], act="swiglu", offsets=off,
                            out=self._h[r], z=self._z[r])
                moe.linear8(*moe.quantise(self._h[r], offsets=off), *self._down8[r][0], offsets=off, out=self._y[r])
            else:
                moe.linear(plan.x, self.up[r], act="swiglu", offsets=off, out=self._h[r], z=self._z[r])
                moe.linear(self._h[r], self.down[r], offsets=off, out=self._y[r])
            moe.combine(self._y[r], plan.rows, weights, out=self._slice(self._scatter, r, n, self.hidden))
            self._saved[r] = (logits, ids, weights)
        self._x = x.clone()
        return self._reduce_scatter()

    def backward(self, dout: torch.Tensor):
        """Gradients of the last forward pass: (dx [P, tokens, hidden], router
        [E, H] float32, up, down: lists of float32 like the weights)."""
        n = self.nranks * self.tokens
        ups, downs, dys = [], [], []
        for r, douts in enumerate(self._all_gather(dout)):
            plan, (_, _, weights) = self.plans[r], self._saved[r]
            dys.append(moe.combine_grad(douts, self._y[r], plan.rows, weights))
        for r, xs in enumerate(self._all_gather(self._x)):
            plan, (logits, ids, weights) = self.plans[r], self._saved[r]
            dy, dweights = dys[r]
            off = plan.offsets
            if self.products == "e4m3":
                dh = moe.linear8(*moe.quantise(dy, offsets=off), *self._down8[r][1], offsets=off, dtype=self.dtype)
                dz = moe.act_grad(dh, self._z[r], "swiglu")
            else:
                dz = moe.linear_grad_x(dy, self.down[r], act="swiglu", z=self._z[r], offsets=off)
            ddown = torch.empty(self.down[r].shape, dtype=torch.float32, device=xs.device)
            moe.linear_grad_w(dy, self._h[r], offsets=off, out=ddown)
            dup = torch.empty(self.up[r].shape, dtype=torch.float32, device=xs.device)
            moe.linear_grad_w(dz, plan.x, offsets=off, out=dup)
            # a rank has the weights' gradient of its own experts' choices only,
            # and the routing gradient is linear in it: the ranks' parts add up
            dlogits = moe.route_grad(logits, ids, dweights, normalise=True)
            moe.linear_grad_w(dlogits, xs.float(), out=self._slice(self._sum, r, *self.router.shape))
            through = moe.linear_grad_x(dlogits, self.router.float()).to(self.dtype)
            if self.products == "e4m3":
                drows = moe.linear8(*moe.quantise(dz, offsets=off), *self._up8[r][1], offsets=off, dtype=self.dtype)
            else:
                drows = moe.linear_grad_x(dz, self.up[r], offsets=off)
            moe.combine(drows, plan.rows, residual=through, out=self._slice(self._scatter, r, n, self.hidden))
            ups.append(dup)
            downs.append(ddown)
        dx = self._reduce_scatter()
        ll.check(self._sum.allreduce(self.router.numel()), "ll_allreduce")
        return dx, self._out(self._sum, 0, *self.router.shape).clone(), ups, downs


class ExpertBlock:
    """The layer between two norms, on a residual stream:

        out = x + scale * post * unit(layer(pre * unit(x)))

    unit(v) = v / sqrt(mean(v^2) + eps).  ``layer`` is an ExpertLayer; ``pre`` and
    ``post`` [hidden] are binary32 and start at 1.  ``options`` are those of
    ``optim.AdamW`` (``floor`` is on unless they say otherwise).  The block updates the
    tensors that it and the layer have when it is made: assign others before; ``step``
    refuses others.  After other values were copied into them call
    ``optimiser.read_params()`` and the layer's ``quantise_weights()``."""

    def __init__(self, layer: ExpertLayer, scale: float = 1.0, eps: float = 1e-6, **options):
        self.layer, self.scale, self.eps = layer, scale, eps
        device = layer.router.device
        self.pre, self.post = (torch.ones(layer.hidden, device=device) for _ in range(2))
        self.params = self._present()
        self.optimiser = AdamW(self.params, **{"floor": True, **options})

    def _present(self) -> list:
        """The tensors that forward and backward use now."""
        return [self.pre, self.post, self.layer.router, *self.layer.up, *self.layer.down]

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        """[P, tokens, hidden] -> the same shape.  A token is on one rank, so the
        norms of all ranks are one call."""
        rows = x.reshape(-1, self.layer.hidden)
        h = moe.norm(rows, self.pre, eps=self.eps).h
        y = self.layer.forward(h.view(x.shape)).view(rows.shape)
        self._saved = (rows.clone(), y)
        return moe.norm(y, residual=rows, post=self.post, scale=self.scale, eps=self.eps).r.view(x.shape)

    def backward(self, dout: torch.Tensor):
        """(dx, the gradients of ``params``) of the last forward pass."""
        rows, y = self._saved
        last = moe.norm_grad(None, None, dr=dout.reshape(rows.shape), y=y, post=self.post, scale=self.scale, eps=self.eps)
        dh, drouter, dup, ddown = self.layer.backward(last.dy.view(dout.shape))
        first = moe.norm_grad(dh.view(rows.shape), rows, self.pre, dr=last.dr, eps=self.eps)
        return first.dr.view(dout.shape), [first.dweight, last.dpost, drouter, *dup, *ddown]

    def step(self, grads, *, stream=None, **options) -> None:
        """One update of ``params``, and the codes of the layer's weights behind it on
        the same stream (options: those of ``AdamW.step``)."""
        present = self._present()
        if len(present) != len(self.params) or any(a is not b for a, b in zip(present, self.params)):
            raise ValueError("the layer's or the block's weights are other tensors than those the block was made with: "
                             "make it anew")
        self.optimiser.step(grads, stream=stream, **options)
        self.layer.quantise_weights(stream)


def main() -> None:
    for products, states in (("same", "f32"), ("e4m3", "8bit")):
        block = ExpertBlock(ExpertLayer(8, 128, 2048, 512, 64, 6, products=products), lr=1e-3, states=states)
        x = torch.randn(8, 128, 2048, device="cuda").to(torch.bfloat16)
        marks = [torch.cuda.Event(enable_timing=True) for _ in range(4)]
        for _ in range(2):
            marks[0].record()
            out = block.forward(x)
            marks[1].record()
            _, grads = block.backward(out)
            marks[2].record()
            block.step(grads)
            marks[3].record()
        torch.cuda.synchronize()
        ll.check(ll.ll_check(SymRegion.stream_handle()), "ll_check")
        times = [a.elapsed_time(b) for a, b in zip(marks, marks[1:])]
        print(f"8 ranks x 128 tokens, hidden 2048, 64 experts of 512, 6 a token, products {products}, states {states}: "
              "forward %.2f ms, backward %.2f ms, update %.2f ms" % tuple(times))


if __name__ == "__main__":
    main()
