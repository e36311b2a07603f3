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

One process drives all the ranks here, so what a rank computes is a loop over
ranks; every step of it uses that rank's own buffers only.

    python -m paper_2607_16100_amd.expert_layer      # one training step, timed
"""
from __future__ import annotations

import torch

from . import llcoll as ll
from . import moe
from .region import SymRegion

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


class ExpertLayer:
    """``tokens``: per rank.  Weights are random, scaled by the square root of
    the fan-in; assign ``router`` [E, H] (binary32), ``up`` [P][E/P, 2F, H] and
    ``down`` [P][E/P, H, F] to use others."""

    def __init__(self, nranks: int, tokens: int, hidden: int, ffn: int, experts: int, k: int, dtype: str = "bf16",
                 seed: int = 0, device="cuda"):
        if experts % nranks:
            raise ValueError(f"{experts} experts over {nranks} ranks")
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
            moe.linear(plan.x, self.up[r], act="swiglu", offsets=plan.offsets, out=self._h[r], z=self._z[r])
            moe.linear(self._h[r], self.down[r], offsets=plan.offsets, out=self._y[r])
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
            moe.combine(moe.linear_grad_x(dz, self.up[r], offsets=off), plan.rows, residual=through,
                        out=self._slice(self._scatter, r, n, self.hidden))
            ups.append(dup)
            downs.append(ddown)
        dx = self._reduce_scatter()
        ll.check(self._sum.allreduce(self.router.numel()), "ll_allreduce")
        return dx, self._out(self._sum, 0, *self.router.shape).clone(), ups, downs


def main() -> None:
    layer = ExpertLayer(8, 128, 2048, 512, 64, 6)
    x = torch.randn(8, 128, 2048, device="cuda").to(torch.bfloat16)
    out = layer.forward(x)
    layer.backward(out)
    ll.check(ll.ll_check(SymRegion.stream_handle()), "ll_check")
    start, mid, end = (torch.cuda.Event(enable_timing=True) for _ in range(3))
    start.record()
    out = layer.forward(x)
    mid.record()
    layer.backward(out)
    end.record()
    torch.cuda.synchronize()
    print(f"8 ranks x 128 tokens, hidden 2048, 64 experts of 512, 6 a token: forward {start.elapsed_time(mid):.2f} ms, "
          f"backward {mid.elapsed_time(end):.2f} ms")


if __name__ == "__main__":
    main()
