"""The weight update of parameters whose memory or values have changed since the
step before."""
from __future__ import annotations

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

if not torch.cuda.is_available():  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

from paper_2607_16100_amd.optim import AdamW  # noqa: E402
from test_moe_gpu import gen, randn  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda"
OPTS = dict(lr=3e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_other_sizes_strides_and_types_at_the_same_address_are_refused(states):
    """Where the memory is the old one a step looks at the parameter all the same."""
    p, grad = randn(gen(1), 64, 64), randn(gen(2), 64, 64)
    opt = AdamW([p], states=states, **OPTS)
    opt.step([grad])
    old, kept = p.data, p.clone()
    for other in (old.t(), old[:32], old.view(BF16)[:, :64], old.view(BF16).reshape(-1)[:64 * 64], old.view(torch.int32)):
        assert other.data_ptr() == old.data_ptr()
        p.data = other
        with pytest.raises(ValueError):
            opt.step([grad])
    p.data = old.view(-1)  # the same values in the same order
    assert torch.equal(p, kept.view(-1)) and int(opt.count) == 1
    opt.step([grad])
    assert int(opt.count) == 2


def twin_of(opt, p, master, states):
    """A parameter of the values `master` (float32), with an optimiser on a copy of opt's state."""
    state = {k: None if t is None else t.clone() for k, t in opt.state_dict().items() if k != "masters"}
    q = master.to(p.dtype)
    state["masters"] = [None if p.dtype is F32 else master.clone()]
    return q, AdamW([q], states=states, state=state, **OPTS)


@pytest.mark.parametrize("states", ["f32", "8bit"])
@pytest.mark.parametrize("how", ["moved", "moved with other values", "refilled", "refilled through data", "moved at first"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_values_that_are_read_are_the_ones_a_parameter_goes_on_from(dtype, how, states):
    g = gen(3)
    n = 700
    p = randn(g, n, dtype=dtype)
    opt = AdamW([p], states=states, **OPTS)
    if how != "moved at first":
        for _ in range(3):
            opt.step([randn(g, n)])
    exact = (p.clone() if dtype is F32 else opt.masters[0].clone()).float()
    other = randn(g, n, dtype=dtype)
    other[::3] = p[::3]  # a part stays as it is, with the bits that only a master has
    want = torch.where(other == p, exact, other.float())
    if how == "moved":
        p.data, want = p.data.clone(), exact
    elif how in ("moved with other values", "moved at first"):
        p.data = other.clone()
    else:
        (p.data if how == "refilled through data" else p).copy_(other)
    opt.read_params()
    q, twin = twin_of(opt, p, want, states)
    grad = randn(g, n)
    opt.step([grad])
    twin.step([grad])
    assert torch.equal(p, q)
    if dtype is BF16:
        assert torch.equal(opt.masters[0], twin.masters[0]) and torch.equal(p, opt.masters[0].to(BF16))


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_a_bfloat16_parameter_is_written_from_its_master(states):
    """Whatever its memory holds, and wherever it is, if nobody says that it should be read."""
    g = gen(6)
    p, grad = randn(g, 700, dtype=BF16), randn(g, 700)
    opt = AdamW([p], states=states, **OPTS)
    opt.step([grad])
    q, twin = twin_of(opt, p, opt.masters[0], states)
    p.data = torch.full_like(p, float("nan"))
    for _ in range(2):
        opt.step([grad])
        twin.step([grad])
        assert torch.equal(p, q) and torch.equal(opt.masters[0], twin.masters[0])
        p.zero_()


def test_parameters_are_read_on_a_side_stream_and_in_a_graph():
    g = gen(4)
    p, fixed = randn(g, 500, dtype=BF16), randn(g, 300, dtype=BF16)
    opt = AdamW([p, fixed], **OPTS)
    opt.step([randn(g, 500), randn(g, 300)])
    grads = [randn(g, 500), randn(g, 300)]
    other = randn(g, 500, dtype=BF16)
    state = {k: [w.clone() for w in t] if k == "masters" else None if t is None else t.clone()
             for k, t in opt.state_dict().items()}
    state["masters"][0] = other.float()
    q = [other.clone(), fixed.clone()]
    twin = AdamW(q, state=state, **OPTS)
    p.data = other.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.read_params()
        opt.step(grads)
    for _ in range(4):
        graph.replay()
        twin.step(grads)
        torch.cuda.synchronize()
        assert torch.equal(p, q[0]) and torch.equal(fixed, q[1])
        assert all(torch.equal(a, b) for a, b in zip(opt.masters, twin.masters))
    # and on a stream of its own, behind what fills the parameter there
    later = torch.empty_like(other)
    big = torch.ones(2048, 2048, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            big = (big @ big).clamp(0, 1)
        later.copy_(other)
    p.data = later
    opt.read_params(side)
    opt.step(grads, stream=side)
    side.synchronize()
    q[0].copy_(other)
    twin.read_params()
    twin.step(grads)
    torch.cuda.synchronize()
    assert torch.equal(p, q[0]) and torch.equal(fixed, q[1])


def test_no_number_in_a_parameter_stays():
    p = torch.ones(10, dtype=BF16, device=DEV)
    opt = AdamW([p], **OPTS)
    p[3], p[5] = float("nan"), float("inf")
    opt.read_params()
    opt.step([torch.ones(10, device=DEV)])
    assert torch.isfinite(p).sum() == 8 and bool(p[3].isnan()) and bool(p[5].isinf())

