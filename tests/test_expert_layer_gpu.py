"""The expert layer over the virtual ranks against the same layer written in
64 bits with torch's autograd."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import moeref as ref  # noqa: E402
from test_moe_gpu import gen, randn  # noqa: E402

if torch.cuda.is_available():
    from paper_2607_16100_amd import llcoll as ll  # noqa: E402
    from paper_2607_16100_amd.expert_layer import ExpertLayer  # noqa: E402
    from paper_2607_16100_amd.region import SymRegion  # noqa: E402
else:  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)


def plain(x, router, up, down, k):
    """The layer on all tokens and experts, float64."""
    p = torch.softmax(x @ router.t(), 1)
    ids = p.topk(k, 1).indices
    w = p.gather(1, ids)
    w = w / w.sum(1, keepdim=True)
    out = torch.zeros_like(x)
    for e in range(router.shape[0]):
        t, j = (ids == e).nonzero(as_tuple=True)
        gate, u = (x[t] @ up[e].t()).chunk(2, 1)
        out = out.index_add(0, t, w[t, j, None] * ((gate * torch.sigmoid(gate) * u) @ down[e].t()))
    return out


@pytest.mark.parametrize("p,tokens,hidden,ffn,experts,k", [(4, 24, 64, 48, 16, 4), (8, 5, 72, 20, 8, 2),
                                                           (2, 70, 40, 33, 6, 6)])
def test_layer_and_gradients(p, tokens, hidden, ffn, experts, k):
    layer = ExpertLayer(p, tokens, hidden, ffn, experts, k, dtype="f32", seed=3)
    g = gen(p)
    x, dout = randn(g, p, tokens, hidden), randn(g, p, tokens, hidden)
    leaves = [x.double().reshape(-1, hidden), layer.router.double(), torch.cat(layer.up).double(),
              torch.cat(layer.down).double()]
    for leaf in leaves:
        leaf.requires_grad_(True)
    want = plain(*leaves, k)
    want.backward(dout.double().reshape(-1, hidden))

    out = layer.forward(x)
    dx, drouter, dup, ddown = layer.backward(dout)
    assert ll.ll_check(SymRegion.stream_handle()) == ll.LL_OK
    # Relative to the largest value: each of the at most eight sums on the way
    # is of no more than `terms` products, in binary32.
    terms = p * tokens * k + hidden + 2 * ffn + experts
    for got, exact in ((out, want), (dx, leaves[0].grad), (drouter, leaves[1].grad), (torch.cat(dup), leaves[2].grad),
                       (torch.cat(ddown), leaves[3].grad)):
        exact = exact.detach().reshape(got.shape)
        err = float((got.double() - exact).abs().max() / exact.abs().max())
        assert err <= 8 * terms * ref.EPS


def test_every_rank_gathers_and_scatters_the_same_layer_in_bfloat16():
    """Two passes of one layer give the same bits, and other tokens other ones."""
    layer = ExpertLayer(8, 16, 256, 64, 32, 4)
    x = randn(gen(1), 8, 16, 256, dtype=torch.bfloat16)
    first = layer.forward(x)
    assert torch.equal(layer.forward(x), first)
    assert not torch.equal(layer.forward(x.flip(0)), first)
    assert torch.equal(layer.forward(x.flip(0)), layer.forward(x.flip(0)))


def test_experts_must_divide():
    with pytest.raises(ValueError):
        ExpertLayer(4, 8, 64, 32, 6, 2)


def in_bfloat16(p, tokens, hidden, ffn, experts, k):
    """A bfloat16 layer, its inputs, and the same layer in 64 bits on the experts it chose."""
    layer = ExpertLayer(p, tokens, hidden, ffn, experts, k, seed=5)
    g = gen(p + 40)
    x, dout = (randn(g, p, tokens, hidden, dtype=torch.bfloat16) for _ in range(2))
    out = layer.forward(x)
    ids = layer._saved[0][1].long()
    leaves = [x.double().reshape(-1, hidden), layer.router.double(), torch.cat(layer.up).double(),
              torch.cat(layer.down).double()]
    for leaf in leaves:
        leaf.requires_grad_(True)
    xs, router, up, down = leaves
    w = torch.softmax(xs @ router.t(), 1).gather(1, ids)
    w = w / w.sum(1, keepdim=True)
    want = torch.zeros_like(xs)
    for e in range(experts):
        t, j = (ids == e).nonzero(as_tuple=True)
        gate, u = (xs[t] @ up[e].t()).chunk(2, 1)
        want = want.index_add(0, t, w[t, j, None] * ((gate * torch.sigmoid(gate) * u) @ down[e].t()))
    want.backward(dout.double().reshape(-1, hidden))
    return layer, x, dout, out, want, leaves


@pytest.mark.parametrize("p,tokens,hidden,ffn,experts,k", [(8, 16, 256, 64, 32, 4), (4, 50, 200, 96, 8, 2)])
def test_bfloat16_layer_and_gradients(p, tokens, hidden, ffn, experts, k):
    """Relative in the Frobenius norm.  A value rounded to bfloat16 is off by at
    most 2^-9 of itself, and the matrices pass a rounding on with at most twice
    the gain (spectral over root-mean-square gain of a random matrix) that the
    values themselves have; what goes through two of them, four times."""
    layer, x, dout, out, want, leaves = in_bfloat16(p, tokens, hidden, ffn, experts, k)
    dx, drouter, dup, ddown = layer.backward(dout)
    assert ll.ll_check(SymRegion.stream_handle()) == ll.LL_OK
    unit = 2.0 ** -9
    # out: h (through one product), y, the ranks' parts, their sum
    # ddown: dy and h.  dup: dy (through one product), the saved z (through the
    # slopes, at most twice), dz.  dx: dup's and the product's own result, the
    # router's share, the ranks' parts and their sum, all but the last two through
    # one product more.  drouter: dweights from y's rounding and h's behind it;
    # the differences g - <u, g> of those are smaller than they are, by up to the
    # two terms' ratio of size, taken as 4.
    for name, got, exact, roundings in (
            ("out", out, want, 2 + 1 + 1 + 1), ("ddown", torch.cat(ddown), leaves[3].grad, 1 + 1),
            ("dup", torch.cat(dup), leaves[2].grad, 2 + 2 + 1),
            ("dx", dx, leaves[0].grad, 4 + 4 + 2 + 1 + 1 + 1 + 1),
            ("drouter", drouter, leaves[1].grad, 4 * (1 + 2) + 1)):
        exact = exact.detach().reshape(got.shape)
        err = float((got.double() - exact).norm() / exact.norm())
        assert err <= roundings * unit, (name, err / unit)


def test_inputs_that_require_gradients_are_refused():
    layer = ExpertLayer(2, 4, 16, 8, 4, 2, dtype="f32")
    x = randn(gen(2), 2, 4, 16)
    want = layer.forward(x)
    x.requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        layer.forward(x)
    with torch.no_grad():
        assert torch.equal(layer.forward(x), want)


@pytest.mark.parametrize("p,tokens,hidden,ffn,experts,k", [(8, 16, 256, 64, 32, 4), (4, 50, 200, 96, 8, 2)])
def test_router_of_a_bfloat16_layer_is_binary32(p, tokens, hidden, ffn, experts, k):
    """Logits, choice, weights and the router's gradient are not rounded to bfloat16."""
    layer = ExpertLayer(p, tokens, hidden, ffn, experts, k, seed=6)
    assert layer.router.dtype is torch.float32
    x = randn(gen(41), p, tokens, hidden, dtype=torch.bfloat16)
    layer.forward(x)
    xs = x.double().reshape(-1, hidden)
    z, ez = ref.matmul(xs, layer.router.double().t())
    for logits, ids, weights in layer._saved:
        ref.close(logits, z, ez, torch.float32)
        u = torch.softmax(z, 1).gather(1, ids.long())
        # an exponential of a logit that is off by ez, shared by a sum of k
        rel = 2 * ez.max() + (k + 48) * ref.EPS
        ref.close(weights, u / u.sum(1, keepdim=True), rel * torch.ones_like(u), torch.float32)
        # no expert left out has a larger logit than one chosen, but for its error
        rest = z.scatter(1, ids.long(), float("-inf")).max(1).values
        assert bool((z.gather(1, ids.long()).min(1).values >= rest - 2 * ez.max()).all())
