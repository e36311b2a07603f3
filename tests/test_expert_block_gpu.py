"""The expert layer with 8-bit products, and the block of norms, layer and
update around it, against the same written in 64 bits with torch's autograd."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import moeref as ref  # noqa: E402
from test_expert_layer_gpu import plain  # noqa: E402
from test_moe_gpu import gen, randn  # noqa: E402

if torch.cuda.is_available():
    from paper_2607_16100_amd import llcoll as ll  # noqa: E402
    from paper_2607_16100_amd import moe  # noqa: E402
    from paper_2607_16100_amd.expert_layer import ExpertBlock, ExpertLayer  # noqa: E402
    from paper_2607_16100_amd.region import SymRegion  # noqa: E402
else:  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

DEV = "cuda"


def unit(x, eps):
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)


@pytest.mark.parametrize("p,tokens,hidden,ffn,experts,k", [(4, 24, 64, 48, 16, 4), (2, 70, 40, 33, 6, 6)])
def test_block_and_gradients(p, tokens, hidden, ffn, experts, k):
    block = ExpertBlock(ExpertLayer(p, tokens, hidden, ffn, experts, k, dtype="f32", seed=3), scale=0.5, eps=1e-5, lr=1e-3)
    layer = block.layer
    g = gen(p)
    block.pre.copy_(1 + 0.3 * randn(g, hidden))
    block.post.copy_(1 + 0.3 * randn(g, hidden))
    x, dout = randn(g, p, tokens, hidden), randn(g, p, tokens, hidden)
    leaves = [x.double().reshape(-1, hidden), block.pre.double(), block.post.double(), layer.router.double(),
              torch.cat(layer.up).double(), torch.cat(layer.down).double()]
    for leaf in leaves:
        leaf.requires_grad_(True)
    xs, pre, post, router, up, down = leaves
    want = xs + 0.5 * post * unit(plain(pre * unit(xs, 1e-5), router, up, down, k), 1e-5)
    want.backward(dout.double().reshape(-1, hidden))
    out = block.forward(x)
    dx, grads = block.backward(dout)
    assert ll.ll_check(SymRegion.stream_handle()) == ll.LL_OK
    got = [dx, grads[0], grads[1], grads[2], torch.cat(grads[3:3 + p]), torch.cat(grads[3 + p:])]
    # Relative to the largest value: of the at most a dozen sums on the way each
    # is of no more than `terms` products, in binary32.
    terms = p * tokens * k + hidden + 2 * ffn + experts
    for a, exact in [(out, want), *((t, leaf.grad) for t, leaf in zip(got, leaves))]:
        exact = exact.detach().reshape(a.shape)
        err = float((a.double() - exact).abs().max() / exact.abs().max())
        assert err <= 12 * terms * ref.EPS

    # the update: one step from states of zero moves a value by lr m / (sqrt(v) + eps) of its own gradient
    before = [t.clone() for t in block.params]
    block.step(grads)
    for old, new, gr in zip(before, block.params, grads):
        gr = gr.double().reshape(old.shape)
        moved = old.double() - 1e-3 * gr / (gr.abs() + 1e-8)
        # (steps of 1e-3, and beta and lr in binary32; gradients under 1e-18 have squares that underflow)
        big = gr.abs() > 1e-15
        assert bool(((new.double() - moved).abs() <= 2 * ref.EPS * old.double().abs() + 1e-3 * 16 * ref.EPS)[big].all())


def layer_by_hand(layer, x, dout):
    """The same calls on one rank's tokens and all ranks' experts, one rank after the other."""
    p, hidden = layer.nranks, layer.hidden
    rows = x.reshape(-1, hidden)
    outs, dxs = [], []
    for r in range(p):
        logits = moe.linear(rows.float(), layer.router)
        ids, weights = moe.route(logits, layer.k, normalise=True)
        plan = moe.Dispatch(rows.shape[0], layer.k, layer.local, hidden, layer.dtype, first=r * layer.local).dispatch(ids, rows)
        off = plan.offsets
        n = int(off[-1])
        z = torch.zeros(rows.shape[0] * layer.k, layer.up[r].shape[1], dtype=layer.dtype, device=DEV)
        h = moe.linear8(*moe.quantise(plan.x, offsets=off), *moe.quantise_weight(layer.up[r]), act="swiglu", offsets=off, z=z,
                        dtype=layer.dtype)
        h[n:] = 0
        y = moe.linear8(*moe.quantise(h), *moe.quantise_weight(layer.down[r]), offsets=off, dtype=layer.dtype)
        outs.append(moe.combine(y, plan.rows, weights))
        dy, dweights = moe.combine_grad(dout.reshape(-1, hidden), y, plan.rows, weights)
        dh = moe.linear8(*moe.quantise(dy), *moe.quantise_weight(layer.down[r], transpose=True), offsets=off, dtype=layer.dtype)
        dh[n:] = 0
        dz = moe.act_grad(dh, z, "swiglu")
        drows = moe.linear8(*moe.quantise(dz), *moe.quantise_weight(layer.up[r], transpose=True), offsets=off,
                            dtype=layer.dtype)
        dlogits = moe.route_grad(logits, ids, dweights, normalise=True)
        through = moe.linear_grad_x(dlogits, layer.router).to(layer.dtype)
        dxs.append(moe.combine(drows, plan.rows, residual=through))
    return outs, dxs


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_layer_with_8_bit_products(dtype):
    p, tokens, hidden, ffn, experts, k = 4, 24, 192, 144, 16, 4
    layer = ExpertLayer(p, tokens, hidden, ffn, experts, k, dtype=dtype, seed=3, products="e4m3")
    same = ExpertLayer(p, tokens, hidden, ffn, experts, k, dtype=dtype, seed=3)
    g = gen(5)
    x, dout = randn(g, p, tokens, hidden, dtype=layer.dtype), randn(g, p, tokens, hidden, dtype=layer.dtype)
    out, near = layer.forward(x), same.forward(x)
    back, plain_back = layer.backward(dout), same.backward(dout)
    assert ll.ll_check(SymRegion.stream_handle()) == ll.LL_OK
    outs, dxs = layer_by_hand(layer, x, dout)
    # the ranks' parts are added in order in binary32 and rounded once
    for got, parts in ((out, outs), (back[0], dxs)):
        total = parts[0].float()
        for t in parts[1:]:
            total = total + t.float()
        assert torch.equal(got.reshape(-1, hidden), total.to(layer.dtype))
    # near the layer without them: two operands off by 2^-4 at most in each of two
    # products, and the gated activation multiplies two of the first one's results
    for a, b in ((out, near), (back[0], plain_back[0]), (torch.cat(back[2]), torch.cat(plain_back[2]))):
        a, b = a.double(), b.double()
        assert float((a - b).norm() / b.norm()) <= 3 * 2 * 2.0 ** -4


def test_updates_reach_the_codes():
    layer = ExpertLayer(2, 16, 128, 64, 4, 2, seed=1, products="e4m3")
    block = ExpertBlock(layer, lr=1e-2, states="8bit", seed=9)
    x = randn(gen(2), 2, 16, 128, dtype=torch.bfloat16)
    for _ in range(3):
        block.step(block.backward(block.forward(x))[1])
    assert int(block.optimiser.count) == 3
    for held, ws in ((layer._up8, layer.up), (layer._down8, layer.down)):
        for ((q, s), (qt, st)), w in zip(held, ws):
            for have, want in (((q, s), moe.quantise_weight(w)), ((qt, st), moe.quantise_weight(w, transpose=True))):
                assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(have, want))
    for w, m in zip(block.params, block.optimiser.masters):
        assert bool(torch.isfinite(w.float()).all()) and (m is None or torch.equal(w, m.to(w.dtype)))


def test_refusals():
    with pytest.raises(ValueError):
        ExpertLayer(2, 4, 16, 8, 4, 2, products="int8")
