"""Steps of a block beside other work, and of a block whose tensors have changed."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_16100_amd import moe  # noqa: E402
from paper_2607_16100_amd.expert_layer import ExpertBlock, ExpertLayer  # noqa: E402
from test_moe_gpu import gen, randn  # noqa: E402

DEV = "cuda"


def make(products="e4m3", states="8bit"):
    return ExpertBlock(ExpertLayer(2, 16, 128, 64, 4, 2, seed=1, products=products), lr=1e-2, states=states, seed=9)


def grads_of(block, seed):
    g = gen(seed)
    return [randn(g, *p.shape) for p in block.params]


def codes_are_the_weights(layer):
    for held, ws in ((layer._up8, layer.up), (layer._down8, layer.down)):
        for ((q, s), (qt, st)), w in zip(held, ws):
            for have, want in (((q, s), moe.quantise_weight(w)), ((qt, st), moe.quantise_weight(w, transpose=True))):
                assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(have, want))


def test_a_step_on_a_busy_side_stream():
    """The update waits behind the stream's other work, and the codes behind the update."""
    a, b = make(), make()
    side = torch.cuda.Stream()
    big = torch.ones(2048, 2048, device=DEV)
    for seed in range(3):
        grads = grads_of(a, seed)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(20):
                big = (big @ big).clamp(0, 1)
        a.step(grads, stream=side)
        b.step(grads)
        side.synchronize()
        torch.cuda.synchronize()
        for x, y in zip(a.params, b.params):
            assert torch.equal(x, y)
        codes_are_the_weights(a.layer)
        codes_are_the_weights(b.layer)


def test_other_weights_than_the_blocks_own():
    """Assigned before the block is made they are updated; behind that a step is refused."""
    layer = ExpertLayer(2, 16, 128, 64, 4, 2, seed=1)
    layer.up = [w.clone() for w in layer.up]
    block = ExpertBlock(layer, lr=1e-2)
    before = [w.clone() for w in layer.up]
    block.step(grads_of(block, 1))
    assert not any(torch.equal(a, b) for a, b in zip(before, layer.up))
    layer.down[1] = layer.down[1].clone()
    kept = [p.clone() for p in block.params]
    with pytest.raises(ValueError):
        block.step(grads_of(block, 2))
    assert all(torch.equal(a, b) for a, b in zip(kept, block.params)) and int(block.optimiser.count) == 1


def test_values_copied_into_the_blocks_weights():
    """A step goes on from them once they are read."""
    a = make()
    a.step(grads_of(a, 1))
    g = gen(8)
    for w in a.params:
        w.copy_(randn(g, *w.shape) * 0.1)
    a.optimiser.read_params()
    a.layer.quantise_weights()
    codes_are_the_weights(a.layer)
    before = [w.clone() for w in a.params]
    a.step(grads_of(a, 2), lr=0.0)
    assert all(torch.equal(x, y) for x, y in zip(before, a.params))
    codes_are_the_weights(a.layer)
