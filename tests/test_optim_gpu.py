"""The weight update on the GPU: binary32 states against 64 bits, 8-bit states
bit for bit against the same operations in numpy."""
from __future__ import annotations

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import blockref as bref  # noqa: E402
import moeref as ref  # noqa: E402
from test_moe_gpu import gen, randn  # noqa: E402

if torch.cuda.is_available():
    from paper_2607_16100_amd import llcoll as ll  # noqa: E402
    from paper_2607_16100_amd.optim import AdamW  # noqa: E402
else:  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda"
OPTS = dict(lr=3e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1)
EPS = ref.EPS


def tensors(g, sizes, dtypes):
    return [randn(g, *(s if isinstance(s, tuple) else (s,)), dtype=dt) for s, dt in zip(sizes, dtypes)]


# more tensors than one launch takes, empty ones, ends inside a block and a chunk
SIZES = [1, 0, 7, 127, 128, 129, 4096, 4097, (33, 65), 20000, 3] + [5 + i for i in range(45)] + [(64, 200), 12288]
DTYPES = [BF16 if i % 3 == 1 else F32 for i in range(len(SIZES))]
GRADS = [BF16 if i % 4 == 2 else F32 for i in range(len(SIZES))]


def reference(p, m, v, g, t, lr, gs=1.0):
    """(p, its error, m, its error, v, its error) in float64.  m and v: two products and a sum,
    2 EPS of their magnitudes (constants rounded once); p: the quotient's operands to a few EPS."""
    b1, b2 = OPTS["betas"]
    g = g * gs
    em = 3 * EPS * (b1 * m.abs() + (1 - b1) * g.abs())
    ev = 4 * EPS * (b2 * v + (1 - b2) * g * g)
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    den = torch.sqrt(v / (1 - b2 ** t)) + OPTS["eps"]
    step = lr / (1 - b1 ** t) * m / den
    # (v may underflow: gradients below 1e-19 have squares that binary32 holds with fewer bits or not)
    q = p * (1 - lr * OPTS["weight_decay"]) - step
    eq = 3 * EPS * p.abs() + lr / (1 - b1 ** t) * em / den + 12 * EPS * step.abs()
    return q, eq, m, em, v, ev


@pytest.mark.parametrize("steps", [1, 5])
def test_states_in_binary32(steps):
    g = gen(steps)
    params = tensors(g, SIZES, DTYPES)
    opt = AdamW(params, **OPTS)
    want = [p.double().reshape(-1) for p in params]
    state = [(torch.zeros_like(w), torch.zeros_like(w)) for w in want]
    for t in range(1, steps + 1):
        grads = [0.1 * x for x in tensors(g, SIZES, GRADS)]
        opt.step(grads)
        assert int(opt.count) == t
        for i, (p, gr) in enumerate(zip(params, grads)):
            n, at = p.numel(), opt.offsets[i]
            m0, v0 = state[i]
            q, eq, m, em, v, ev = reference(want[i], m0, v0, gr.double().reshape(-1), t, OPTS["lr"])
            got_m, got_v = opt.m[at:at + n], opt.v[at:at + n]
            ref.close(got_m, m, em, F32)
            ref.close(got_v, v, ev, F32)
            master = opt.masters[i]
            exact = p if master is None else master
            ref.close(exact.reshape(-1), q, eq, F32)
            if master is not None:
                assert torch.equal(p, master.to(BF16))
            # go on from what the kernel holds
            want[i] = exact.double().reshape(-1)
            state[i] = (got_m.double(), got_v.double())
            end = (n + 127) // 128 * 128
            assert bool((opt.m[at + n:at + end] == 0).all()) and bool((opt.v[at + n:at + end] == 0).all())


def eight_step(opt, i, n, grad, t, seed, gs=np.float32(1)):
    """(m codes, m scales, v codes, v scales) that the step makes of tensor i's states as they are."""
    at = opt.offsets[i]
    sl, bl = slice(at, at + n), slice(at // 128, (at + n + 127) // 128)
    ms, vs = opt.m_scales[bl].view(torch.uint8).cpu().numpy(), opt.v_scales[bl].view(torch.uint8).cpu().numpy()
    two = lambda c: (c.astype(np.uint32) << 23).view(np.float32)  # noqa: E731
    m = opt.m[sl].float().cpu().numpy() * np.repeat(two(ms), 128)[:n]
    v = opt.v[sl].float().cpu().numpy() * np.repeat(two(vs), 128)[:n]
    m, v = bref.adamw_states(m, v, grad * gs, *OPTS["betas"])
    r = bref.random_bits(at, n, t, seed)
    sm, sv = bref.block_scales(m, 8), bref.block_scales(v, 15)
    mc = bref.stochastic(m, sm, (r >> np.uint64(16)) << np.uint64(4), 3, -6, 7)
    vc = bref.stochastic(v, sv, (r & np.uint64(0xFFFF)) << np.uint64(5), 2, -14, 15)
    return (mc, sm, vc, sv), (m, v)


@pytest.mark.parametrize("seed", [0, 123456789])
def test_states_in_8_bits_bit_for_bit(seed):
    g = gen(7)
    params = tensors(g, SIZES, DTYPES)
    opt = AdamW(params, states="8bit", seed=seed, **OPTS)
    for t in range(1, 5):
        spread = [torch.exp(2 * randn(g, *p.shape)) * 10.0 ** -(i % 6) for i, p in enumerate(params)]
        grads = [(x * s).to(dt) for x, s, dt in zip(tensors(g, SIZES, [F32] * len(SIZES)), spread, GRADS)]
        before = [p.double().reshape(-1) if w is None else w.double().reshape(-1) for p, w in zip(params, opt.masters)]
        want = [eight_step(opt, i, p.numel(), gr.float().cpu().numpy().reshape(-1), t, seed)
                for i, (p, gr) in enumerate(zip(params, grads))]
        opt.step(grads)
        for i, p in enumerate(params):
            n, at = p.numel(), opt.offsets[i]
            (mc, sm, vc, sv), (m, v) = want[i]
            blocks = slice(at // 128, (at + n + 127) // 128)
            assert np.array_equal(opt.m_scales[blocks].view(torch.uint8).cpu().numpy(), sm)
            assert np.array_equal(opt.v_scales[blocks].view(torch.uint8).cpu().numpy(), sv)
            assert np.array_equal(opt.m[at:at + n].view(torch.uint8).cpu().numpy(), mc)
            assert np.array_equal(opt.v[at:at + n].view(torch.uint8).cpu().numpy(), vc)
            end = (n + 127) // 128 * 128
            assert bool((opt.m[at + n:at + end].view(torch.uint8) == 0).all())
            # the parameter moves by the states before they were rounded
            b1, b2 = OPTS["betas"]
            m, v = torch.from_numpy(m).to(DEV).double(), torch.from_numpy(v).to(DEV).double()
            step = OPTS["lr"] / (1 - b1 ** t) * m / (torch.sqrt(v / (1 - b2 ** t)) + OPTS["eps"])
            q = before[i] * (1 - OPTS["lr"] * OPTS["weight_decay"]) - step
            got = p if opt.masters[i] is None else opt.masters[i]
            ref.close(got.reshape(-1), q, 3 * EPS * before[i].abs() + 12 * EPS * step.abs(), F32)


def test_rounding_at_random_keeps_the_mean():
    """A thousand values that are the same: codes on both sides, their mean near
    the value.  The sum of n independent roundings of one step has a variance of
    at most n / 4 steps^2: six deviations of it are 3 / sqrt(n) steps."""
    n = 128 * 512
    p = torch.zeros(n, device=DEV)
    opt = AdamW([p], states="8bit", lr=0.0, betas=(0.9, 0.95))
    grad = torch.full((n,), 0.3, device=DEV)
    grad[::128] = 1.0  # the block's largest
    opt.step([grad])
    got = opt.m.float() * (opt.m_scales.float().repeat_interleave(128))
    rest = torch.ones(n, dtype=torch.bool, device=DEV)
    rest[::128] = False
    values = got[rest].double()
    steps = values.unique()
    assert steps.numel() == 2
    k = values.numel()
    assert abs(float(values.mean()) - 0.1 * float(np.float32(0.3))) <= 3 / math.sqrt(k) * float(steps[1] - steps[0]) + 1e-8


def test_small_changes_are_not_lost():
    """v decays by 5 % a step without gradients; to the nearest code of two bits it would stay."""
    n = 128 * 64
    opt = AdamW([torch.zeros(n, device=DEV)], states="8bit", lr=0.0, betas=(0.9, 0.999))
    first = torch.full((n,), 0.7, device=DEV)
    first[::128] = 1.0
    opt.step([first])

    def mean():
        return float((opt.v.double() * opt.v_scales.double().repeat_interleave(128)).mean())

    start = mean()
    quiet = torch.zeros(n, device=DEV)
    quiet[::128] = 1.0  # keeps the blocks' scale
    for _ in range(200):
        opt.step([quiet])
    others = opt.v.double() * opt.v_scales.double().repeat_interleave(128)
    others[::128] = 0
    # 0.999^200 = 0.82 of the first step's (0.49e-3); a walk of 200 roundings on 8128 values stays within a tenth
    want = 0.49e-3 * 0.999 ** 200 * (127 / 128)
    assert abs(float(others.mean()) - want) <= 0.1 * want
    assert start > 0


def test_learning_rate_and_gradient_scale_from_memory_and_replays():
    g = gen(11)
    sizes = [300, (40, 50), 1]
    for states in ("f32", "8bit"):
        params = tensors(g, sizes, [F32, BF16, F32])
        twin = [p.clone() for p in params]
        a = AdamW(params, states=states, seed=5, **OPTS)
        b = AdamW(twin, states=states, seed=5, **OPTS)
        grads = tensors(g, sizes, [F32, F32, BF16])
        held = [x.clone() for x in grads]
        lr, gs = torch.tensor([0.01], device=DEV), torch.tensor([0.5], device=DEV)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            a.step(held, lr=lr, grad_scale=gs)
        assert int(a.count) == 0
        for t in range(1, 6):
            lr.fill_(0.01 / t)
            gs.fill_(0.5 * t)
            for x, y in zip(held, grads):
                x.copy_(y * t)
            graph.replay()
            b.step(held, lr=float(lr), grad_scale=gs)
            torch.cuda.synchronize()
            assert int(a.count) == t == int(b.count)
            for x, y in zip(params, twin):
                assert torch.equal(x, y)
            for name in ("m", "v"):
                assert torch.equal(getattr(a, name).view(torch.uint8), getattr(b, name).view(torch.uint8))
        if states == "f32":  # the scale is a product in front
            c = [p.clone() for p in twin]
            one, two = AdamW(c, **OPTS), AdamW([p.clone() for p in twin], **OPTS)
            one.step(grads, grad_scale=gs.fill_(0.25))
            two.step([x * 0.25 for x in grads])
            for x, y in zip(one.params, two.params):
                assert torch.equal(x, y)


def test_going_on_from_a_state():
    g = gen(12)
    for states in ("f32", "8bit"):
        params = tensors(g, [500, (30, 40)], [BF16, F32])
        a = AdamW(params, states=states, seed=3, **OPTS)
        a.step(tensors(g, [500, (30, 40)], [F32, F32]))
        kept = {k: [None if w is None else w.clone() for w in t] if isinstance(t, list) else None if t is None else t.clone()
                for k, t in a.state_dict().items()}
        twin = [p.clone() for p in params]
        b = AdamW(twin, states=states, seed=3, state=kept, **OPTS)
        grads = tensors(g, [500, (30, 40)], [F32, BF16])
        a.step(grads)
        b.step(grads)
        for x, y in zip(params, twin):
            assert torch.equal(x, y)
        assert torch.equal(a.m.view(torch.uint8), b.m.view(torch.uint8)) and int(b.count) == 2


def test_parameters_that_move():
    """A parameter whose memory is another one now is updated there; one of another shape or type is refused."""
    g = gen(14)
    p = randn(g, 300)
    opt = AdamW([p], **OPTS)
    old, grad = p.data, randn(g, 300)
    p.data = old.clone()
    opt.step([grad])
    assert not torch.equal(p, old)
    twin = old.clone()
    AdamW([twin], **OPTS).step([grad])
    assert torch.equal(p, twin)
    for other in (torch.zeros(301, device=DEV), torch.zeros(300, dtype=BF16, device=DEV), torch.zeros(600, device=DEV)[::2]):
        p.data = other
        with pytest.raises(ValueError):
            opt.step([grad])
    assert int(opt.count) == 1


def test_unaligned_tensors_and_a_side_stream():
    g = gen(13)
    for states in ("f32", "8bit"):
        buf = torch.zeros(3000, device=DEV)
        p = buf[1:1 + 2500]
        p.copy_(randn(g, 2500))
        twin = p.clone()
        grad = torch.zeros(2600, dtype=BF16, device=DEV)[3:2503]
        grad.copy_(randn(g, 2500))
        a, b = AdamW([p], states=states, **OPTS), AdamW([twin], states=states, **OPTS)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        a.step([grad], stream=side)
        side.synchronize()
        b.step([grad.clone()])
        assert torch.equal(p, twin)
        assert torch.equal(a.m.view(torch.uint8), b.m.view(torch.uint8))
        assert float(buf[0]) == 0 and bool((buf[2501:] == 0).all())


def test_a_gradient_that_is_no_number_stays_where_it_is():
    for states in ("f32", "8bit"):
        p = torch.ones(300, device=DEV)
        opt = AdamW([p], states=states, **OPTS)
        grad = torch.ones(300, device=DEV)
        grad[130], grad[7] = math.nan, math.inf
        opt.step([grad])
        bad = torch.zeros(300, dtype=torch.bool, device=DEV)
        bad[[7, 130]] = True
        assert torch.equal(~torch.isfinite(p), bad)
        assert torch.equal(~torch.isfinite(opt.m[:300].float()), bad)


def test_refusals():
    p = torch.zeros(10, device=DEV)
    for params, kw in (([], {}), ([p, p], {}), ([p.cpu()], {}), ([torch.zeros(4, 4, device=DEV).t()[:, :2]], {}),
                       ([p], dict(states="16"))):
        with pytest.raises(ValueError):
            AdamW(params, **kw)
    with pytest.raises(ll.LLError):
        AdamW([p.half()])
    opt = AdamW([p])
    for grads in ([], [p[:9]], [p.cpu()], [torch.zeros(20, device=DEV)[::2]]):
        with pytest.raises(ValueError):
            opt.step(grads)
    with pytest.raises(ll.LLError):
        opt.step([p.half()])
    with pytest.raises(ValueError):
        opt.step([p.clone()], lr=torch.zeros(2, device=DEV))
    for kw in (dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(eps=0.0), dict(lr=math.nan),
               dict(weight_decay=-1.0)):
        with pytest.raises(ll.LLError):
            AdamW([p], **kw).step([p.clone()])
    state = opt.state_dict()
    with pytest.raises(ValueError):
        AdamW([p, torch.zeros(300, device=DEV)], state=state)
    with pytest.raises(ValueError):
        AdamW([p], states="8bit", state=state)
    assert int(opt.count) == 0


def test_parameters_in_the_same_memory_are_refused():
    flat = torch.zeros(300, device=DEV)
    for params in ([flat[:200], flat[100:]], [flat[100:], flat[:101]], [flat, flat]):
        with pytest.raises(ValueError):
            AdamW(params)
    a, b = flat[:100], flat[100:200]
    opt = AdamW([a, b, flat[200:200]])
    opt.step([torch.ones(100, device=DEV)] * 2 + [torch.ones(0, device=DEV)])
    b.data = flat[50:150]  # moves into the other
    with pytest.raises(ValueError):
        opt.step([torch.ones(100, device=DEV)] * 2 + [torch.ones(0, device=DEV)])


def test_a_backward_pass_behind_a_step_says_so():
    w = torch.ones(8, device=DEV, requires_grad=True)
    loss = (w * w).sum()
    AdamW([w]).step([torch.ones(8, device=DEV)])
    with pytest.raises(RuntimeError):
        loss.backward()
