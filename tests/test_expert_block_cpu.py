"""What a block's step hands on, without a GPU."""
import types

import pytest

torch = pytest.importorskip("torch")

from paper_2607_16100_amd import expert_layer as el  # noqa: E402


def make(products="e4m3"):
    """(a block of two ranks on CPU tensors, the calls it makes)."""
    calls = []
    layer = object.__new__(el.ExpertLayer)
    layer.products, layer._up8, layer._down8 = products, None, None
    layer.router = torch.zeros(4, 8)
    layer.up, layer.down = ([torch.zeros(2, 6, 8) for _ in range(2)] for _ in range(2))
    block = object.__new__(el.ExpertBlock)
    block.layer = layer
    block.pre, block.post = torch.ones(8), torch.ones(8)
    block.params = [block.pre, block.post, layer.router, *layer.up, *layer.down]
    block.optimiser = types.SimpleNamespace(step=lambda grads, **kw: calls.append(("step", kw)))
    return block, calls


def recorded(monkeypatch, calls):
    def quantise_weight(w, *, transpose=False, out=None, scales=None, stream=None):
        calls.append(("codes", {"stream": stream}))
        return w, w

    monkeypatch.setattr(el.moe, "quantise_weight", quantise_weight)


@pytest.mark.parametrize("stream", [None, "side"])
def test_codes_are_made_on_the_updates_stream(monkeypatch, stream):
    block, calls = make()
    recorded(monkeypatch, calls)
    for _ in range(2):  # the first makes the codes' memory
        calls.clear()
        block.step([], stream=stream, lr=1e-3)
        assert calls[0] == ("step", {"stream": stream, "lr": 1e-3})
        assert calls[1:] == [("codes", {"stream": stream})] * 8


@pytest.mark.parametrize("where", ["router", "up", "down", "pre", "post", "more"])
def test_other_tensors_than_the_blocks_own_are_refused(monkeypatch, where):
    block, calls = make()
    recorded(monkeypatch, calls)
    layer = block.layer
    if where == "router":
        layer.router = layer.router.clone()
    elif where == "up":
        layer.up[1] = layer.up[1].clone()
    elif where == "down":
        layer.down = [w.clone() for w in layer.down]
    elif where == "more":
        layer.up.append(layer.up[0])
    else:
        setattr(block, where, getattr(block, where).clone())
    with pytest.raises(ValueError):
        block.step([])
    assert not calls


def test_the_blocks_own_tensors_in_another_list(monkeypatch):
    block, calls = make("same")
    recorded(monkeypatch, calls)
    block.layer.up = list(block.layer.up)
    block.step([])
    assert calls == [("step", {"stream": None})]
