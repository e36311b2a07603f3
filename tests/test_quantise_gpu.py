"""Rows and weights in 8 bits on the GPU: codes and scales are exact."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import blockref as bref  # noqa: E402
import moeref as ref  # noqa: E402
from test_moe_gpu import gen, randn, strided  # noqa: E402

if torch.cuda.is_available():
    from paper_2607_16100_amd import llcoll as ll  # noqa: E402
    from paper_2607_16100_amd import moe  # noqa: E402
else:  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda"
LAYOUTS = [(0, 0), (3, 1), (8, 0)]  # row padding, first element; NaN in the padding


def hard(g, n, h, dtype):
    """Rows with what a scale can meet: zeros, the smallest and largest values, some that are not finite."""
    x = randn(g, n, h) * torch.exp(3 * randn(g, n, 1))
    if n > 8:
        x[0] = 0
        x[1] *= 1e-38  # subnormal numbers
        x[2] *= 1e37
        x[3, ::7] = math.nan
        x[4, ::5] = math.inf
        x[5, 1::3] = -math.inf
        x[6] = math.nan
        x[7] = x[7].sign() * torch.exp2(torch.randint(-20, 20, (h,), generator=g, device=DEV).float())
        x[8, : h // 2] = 0
    return x.to(dtype)


@pytest.mark.parametrize("n,h", [(1, 1), (1, 128), (3, 129), (11, 127), (17, 256), (9, 1000), (130, 776), (2, 8),
                                 (33, 2048), (1200, 8192)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", [0, 1, 2])
def test_rows(n, h, dtype, layout):
    x = strided(hard(gen(n + h), n, h, dtype), *LAYOUTS[layout])
    q, scales = moe.quantise(x)
    want, codes = bref.quantise(x.double())
    assert torch.equal(scales.view(torch.uint8).long(), codes.long())
    bref.same_values(q, want)


def test_every_bfloat16_value_rounds_to_the_nearest_code():
    """65536 values under a scale of 1, ties among them."""
    x = torch.arange(65536, device=DEV, dtype=torch.int32).to(torch.int16).view(BF16)
    x = torch.where(x.float().abs() <= 448, x, torch.zeros_like(x))
    rows = torch.zeros(65536 // 64, 128, dtype=BF16, device=DEV)
    rows[:, :64] = x.view(-1, 64)
    rows[:, 100] = 448
    q, scales = moe.quantise(rows)
    assert bool((scales.view(torch.uint8) == 127).all())
    bref.same_values(q, bref.round_e4m3(rows.double()))


@pytest.mark.parametrize("act", ["relu", "gelu", "silu", "swiglu", "geglu"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,h,layout", [(1, 40, 0), (70, 264, 1), (33, 1001, 0), (300, 2048, 2)])
def test_activation_in_front(act, dtype, n, h, layout):
    width = 2 * h if act in ref.GATED else h
    x = strided(2 * randn(gen(h), n, width, dtype=dtype), *LAYOUTS[layout])
    q, scales = moe.quantise(x, act=act)
    z = x.double()
    want, err = ref.act(z, act), ref.act_err(z, torch.zeros_like(z), act) + 2.0 ** -126
    s = scales.view(torch.uint8).long()
    amax = torch.stack([p.abs().amax(1) for p in want.split(128, 1)], 1)
    slack = torch.stack([p.amax(1) for p in err.split(128, 1)], 1)
    assert bool(((s >= bref.exponents((amax - slack).clamp(min=0))) & (s <= bref.exponents(amax + slack))).all())
    step = bref.stretch(s, h, 1)
    # half a step of the code: 2^-4 of the value, or half the subnormal step 2^-9
    bound = (err + (want.abs() + err) * 2.0 ** -4).maximum(step * 2.0 ** -10 + err)
    assert bool(((q.double() * step - want).abs() <= bound * 1.0001).all())


@pytest.mark.parametrize("act,h", [("none", 200), ("swiglu", 136)])
def test_rows_behind_the_last_group_are_left(act, h):
    n, used = 70, 37
    x = randn(gen(5), n, 2 * h if act in ref.GATED else h, dtype=BF16)
    x[used:] = math.nan
    off = torch.tensor([0, 5, 5, used], dtype=torch.int32, device=DEV)
    q = torch.full((n, h), 0x35, dtype=torch.uint8, device=DEV).view(moe.E4M3)
    scales = moe.scales_of(n, (h + 127) // 128)
    scales.view(torch.uint8).fill_(77)
    moe.quantise(x, act=act, offsets=off, out=q, scales=scales)
    assert bool((q[used:].view(torch.uint8) == 0x35).all()) and bool((scales[used:].view(torch.uint8) == 77).all())
    alone, s = moe.quantise(x[:used], act=act)
    assert torch.equal(q[:used].view(torch.uint8), alone.view(torch.uint8))
    assert torch.equal(scales[:used].view(torch.uint8), s.view(torch.uint8))


@pytest.mark.parametrize("groups,o,i", [(1, 1, 1), (1, 128, 128), (1, 130, 257), (3, 96, 200), (2, 515, 1001),
                                        (5, 264, 136), (1, 2048, 1024)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pad", [0, 3, 8])
@pytest.mark.parametrize("transpose", [False, True])
def test_weights(groups, o, i, dtype, pad, transpose):
    g = gen(o + i)
    buf = torch.full((groups, o, i + pad), math.nan, dtype=dtype, device=DEV)
    w = buf[:, :, :i]
    w.copy_(randn(g, groups, o, i) * torch.exp(2 * randn(g, groups, o, 1)))
    w[0, :1, :2] = math.inf
    if groups > 1:
        w[1] = 0
    arg = w if groups > 1 else w[0]
    q, scales = moe.quantise_weight(arg, transpose=transpose)
    q, scales = q.view(groups, *q.shape[-2:]), scales.view(torch.uint8).reshape(groups, *scales.shape[-2:])
    for gi in range(groups):
        want, codes = bref.quantise_weight(w[gi].double())
        if transpose:
            want, codes = want.t(), codes.t()
        assert torch.equal(scales[gi].long(), codes.long())
        bref.same_values(q[gi], want)


def test_a_weights_output_with_rows_apart():
    w = randn(gen(1), 2, 150, 140)
    for transpose, (r, c) in ((False, (150, 140)), (True, (140, 150))):
        buf = torch.full((2, r + 2, c + 5), 0x11, dtype=torch.uint8, device=DEV)
        out = buf.view(moe.E4M3)[:, :r, :c]
        q, scales = moe.quantise_weight(w, transpose=transpose, out=out)
        alone, s = moe.quantise_weight(w, transpose=transpose)
        assert torch.equal(q.view(torch.uint8), alone.view(torch.uint8))
        assert torch.equal(scales.view(torch.uint8), s.view(torch.uint8))
        assert bool((buf[:, r:] == 0x11).all()) and bool((buf[:, :, c:] == 0x11).all())


def test_refusals():
    x = torch.zeros(4, 200, device=DEV)
    with pytest.raises(ValueError):
        moe.quantise(x, out=torch.zeros(4, 200, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):  # rows of scales at odd addresses
        moe.quantise(x, scales=torch.zeros(4, 2, dtype=torch.uint8, device=DEV).view(moe.E8M0))
    with pytest.raises(ValueError):
        moe.quantise(x[:, :199], act="swiglu")
    with pytest.raises(ll.LLError):
        moe.quantise(x.half())
    with pytest.raises(ValueError):
        moe.quantise(torch.zeros(4, 200))
    with pytest.raises(ValueError):
        moe.quantise(x, offsets=torch.zeros(0, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        moe.quantise(x.clone().requires_grad_())
    with pytest.raises(ValueError):
        moe.quantise_weight(x.view(2, 2, 200), out=torch.zeros(2, 2, 199, dtype=torch.uint8, device=DEV).view(moe.E4M3))
    q, s = moe.quantise(x[:0])
    assert q.shape == (0, 200) and s.shape == (0, 2)


def test_a_side_stream_and_a_graph():
    x = randn(gen(3), 300, 520, dtype=BF16)
    want, ws = moe.quantise(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    q, s = moe.quantise(x, stream=side)
    side.synchronize()
    assert torch.equal(q.view(torch.uint8), want.view(torch.uint8))
    assert torch.equal(s.view(torch.uint8), ws.view(torch.uint8))
    q, s = torch.zeros_like(want), moe.scales_of(300, 5)
    held = torch.zeros_like(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moe.quantise(held, out=q, scales=s)
    for seed in range(4):
        held.copy_(randn(gen(seed), 300, 520, dtype=BF16))
        graph.replay()
        want, ws = moe.quantise(held)
        torch.cuda.synchronize()
        assert torch.equal(q.view(torch.uint8), want.view(torch.uint8))
        assert torch.equal(s.view(torch.uint8), ws.view(torch.uint8))
