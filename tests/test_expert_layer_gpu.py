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
