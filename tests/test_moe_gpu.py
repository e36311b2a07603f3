"""Routing, dispatch and combine on the GPU against plain 64-bit forms."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import moeref as ref  # noqa: E402

if torch.cuda.is_available():
    from paper_2607_16100_amd import llcoll as ll  # noqa: E402
    from paper_2607_16100_amd import moe  # noqa: E402
else:  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda"


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def strided(t, pad, lead=0):
    """The same matrix with rows `pad` elements further apart, the first one
    `lead` elements into its buffer; NaN in between."""
    n, c = t.shape
    buf = torch.full((n * (c + pad) + lead + 8,), math.nan, dtype=t.dtype, device=t.device)
    v = buf[lead:lead + n * (c + pad)].view(n, c + pad)[:, :c]
    v.copy_(t)
    return v


# ---------------------------------------------------------------- routing
ROUTE = [
    # tokens, experts, k
    (1, 1, 1), (1, 8, 8), (3, 5, 2), (17, 16, 1), (64, 60, 6), (33, 64, 8), (5, 100, 16), (130, 160, 6),
    (19, 256, 8), (7, 257, 4), (3, 1000, 32), (9, 1024, 8), (2, 32, 20), (1025, 128, 8),
]


def route_inputs(t, e, dtype, seed, masked):
    g = gen(seed)
    x = randn(g, t, e) * 1.5
    if masked:
        x[torch.rand(t, e, generator=g, device=DEV) < 0.3] = -math.inf
        x[torch.rand(t, e, generator=g, device=DEV) < 0.05] = math.nan
        x[::3] = -math.inf
        x[1::5, : e // 2] = torch.finfo(dtype).min
    return x.to(dtype)


@pytest.mark.parametrize("t,e,k", ROUTE)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("score,normalise,masked,pad", [
    ("softmax", False, False, 0), ("softmax", True, True, 3), ("sigmoid", False, True, 8), ("sigmoid", True, False, 1)])
def test_route_and_gradient(t, e, k, dtype, score, normalise, masked, pad):
    x = route_inputs(t, e, dtype, t + e, masked)
    bias = 0.3 * randn(gen(e), e) if normalise else None
    v = strided(x, pad)
    ids, w = moe.route(v, k, bias=bias, score=score, normalise=normalise, scale=2.5)
    want_ids, want_w = ref.route(x.double(), bias, k, score, normalise, 2.5)
    assert torch.equal(ids.long(), want_ids)
    # relative: exp of a difference of two logits (|x| of a few units, so a few
    # EPS each), a sum of e positive terms, another of k, two quotients
    rel = (e + k + 48) * ref.EPS
    ref.close(w, want_w, want_w.abs() * rel, F32)

    g = randn(gen(3), t, k)
    got = moe.route_grad(v, ids, g, score=score, normalise=normalise, scale=2.5)
    want = route_grad64(x.double(), want_ids, g.double(), score, normalise, 2.5)
    size = 2.5 * (g.abs() * (want_ids >= 0)).sum(1, keepdim=True).double()
    ref.close(got, want, size * rel * torch.ones_like(want), dtype)


def route_weights64(l, ids, score, normalise, scale):
    l = torch.where(torch.isnan(l), torch.full_like(l, -math.inf), l)
    p = torch.softmax(l, 1).nan_to_num(0.0) if score == "softmax" else torch.sigmoid(l)
    u = torch.where(ids >= 0, p.gather(1, ids.clamp(min=0)), 0.0)
    if normalise:
        tot = u.sum(1, keepdim=True)
        u = torch.where(tot > 0, u / torch.where(tot > 0, tot, 1.0), 0.0)
    return scale * u


def route_grad64(l, ids, g, score, normalise, scale):
    """By the chain rule, written out over all experts."""
    l = torch.where(torch.isnan(l), torch.full_like(l, -math.inf), l)
    p = torch.softmax(l, 1).nan_to_num(0.0) if score == "softmax" else torch.sigmoid(l)
    t, e = l.shape
    chosen = torch.zeros(t, e + 1, dtype=torch.float64, device=DEV)
    up = torch.zeros_like(chosen)
    at = torch.where(ids >= 0, ids, e)
    chosen.scatter_(1, at, 1.0)
    up.scatter_(1, at, scale * g)
    chosen, up = chosen[:, :e], up[:, :e] * chosen[:, :e]
    if normalise:
        tot = (p * chosen).sum(1, keepdim=True)
        safe = torch.where(tot > 0, tot, 1.0)
        up = torch.where(tot > 0, chosen * (up - (up * p).sum(1, keepdim=True) / safe) / safe, 0.0)
    if score == "softmax":
        return p * (up - (up * p).sum(1, keepdim=True))
    return up * p * (1 - p)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("normalise", [False, True])
def test_route_gradient_against_differences(score, normalise):
    t, e, k = 6, 24, 4
    x = randn(gen(5), t, e)
    g = randn(gen(6), t, k)
    ids, _ = moe.route(x, k, score=score, normalise=normalise)
    got = moe.route_grad(x, ids, g, score=score, normalise=normalise).double()
    h = 1e-5  # second-order error h^2, rounding 1e-16 / h: both far below 1e-8
    for i in range(e):
        hi, lo = x.double().clone(), x.double().clone()
        hi[:, i] += h
        lo[:, i] -= h
        d = (route_weights64(hi, ids.long(), score, normalise, 1.0)
             - route_weights64(lo, ids.long(), score, normalise, 1.0)) * g.double()
        num = d.sum(1) / (2 * h)
        assert torch.all((got[:, i] - num).abs() <= 1e-8 + 100 * ref.EPS * g.abs().sum(1))


def test_route_ties_go_to_the_lowest_index():
    for e in (16, 60, 256, 1024):
        x = torch.zeros(5, e, device=DEV)
        x[1, e // 2:] = 1.0
        x[2] = -0.0
        x[2, 3] = 0.0  # equal to -0
        x[3, 1::2] = -math.inf
        x[4] = math.inf
        ids, _ = moe.route(x, 4)
        assert ids[0].tolist() == [0, 1, 2, 3]
        assert ids[1].tolist() == [e // 2 + i for i in range(4)]
        assert ids[2].tolist() == [0, 1, 2, 3]
        assert ids[3].tolist() == [0, 2, 4, 6]
        assert ids[4].tolist() == [0, 1, 2, 3]


def test_route_gradient_skips_ids_out_of_range():
    x = randn(gen(1), 3, 16)
    ids = torch.tensor([[-1, 3], [16, 2], [-5, 1 << 30]], dtype=torch.int32, device=DEV)
    g = torch.ones(3, 2, device=DEV)
    got = moe.route_grad(x, ids, g, score="sigmoid")
    want = torch.zeros(3, 16, dtype=torch.float64, device=DEV)
    s = torch.sigmoid(x.double())
    want[0, 3], want[1, 2] = (s * (1 - s))[0, 3], (s * (1 - s))[1, 2]
    ref.close(got, want, want.abs() * 40 * ref.EPS, F32)


# ---------------------------------------------------------------- dispatch
DISPATCH = [
    # tokens, k, experts in all, first, local, features
    (0, 2, 8, 0, 8, 64), (1, 1, 1, 0, 1, 8), (1, 8, 256, 32, 32, 7168), (16, 8, 256, 224, 32, 512),
    (37, 6, 60, 0, 60, 100), (128, 8, 64, 8, 8, 33), (129, 8, 64, 8, 8, 264), (700, 4, 1024, 0, 1024, 64),
    (1500, 2, 16, 15, 1, 2056), (3000, 1, 8, 6, 4, 16), (5001, 6, 160, 40, 80, 72), (2048, 32, 300, 7, 290, 8),
]


@pytest.mark.parametrize("t,k,e,first,local,h", DISPATCH)
@pytest.mark.parametrize("dtype,pad,lead", [(BF16, 0, 0), (F32, 3, 1), (BF16, 8, 8)])
def test_dispatch(t, k, e, first, local, h, dtype, pad, lead):
    g = gen(t + k)
    ids = torch.randint(-1, e, (t, k), generator=g, device=DEV, dtype=torch.int32)
    x = strided(randn(g, t, h, dtype=dtype), pad, lead)
    plan = moe.Dispatch(t + 5, k, local, h, dtype, first=first)
    plan._x.fill_(7.0)
    plan._slots.fill_(99)
    plan.dispatch(ids, x)
    offsets, slots, rows = ref.sort(ids, first, local)
    assert plan.offsets.tolist() == offsets
    assert plan.slots.tolist() == slots
    assert torch.equal(plan.rows.cpu(), rows)
    n = offsets[-1]
    if n:
        src = torch.tensor(slots[:n], device=DEV) // k
        assert torch.equal(plan.x[:n], x[src])
    assert bool((plan._x[n:] == 7.0).all())  # rows past the last are left alone
    assert plan._slots[t * k:].tolist() == [99] * (5 * k)


def test_dispatch_sort_only_and_its_gradient():
    g = gen(4)
    ids = torch.randint(0, 16, (300, 4), generator=g, device=DEV, dtype=torch.int32)
    plan = moe.Dispatch(300, 4, 8, 40, F32, first=4)
    plan.dispatch(ids)
    assert torch.equal(plan.rows.cpu(), ref.sort(ids, 4, 8)[2])
    dx = randn(g, 1200, 40)
    got = plan.grad(dx)
    ok = plan.rows >= 0
    picked = torch.where(ok[..., None], dx.double()[plan.rows.clamp(min=0).long()], 0.0)
    ref.close(got, picked.sum(1), 6 * ref.EPS * picked.abs().sum(1), F32)


def test_dispatch_every_token_to_one_expert_and_none():
    for t in (50, 4000):
        ids = torch.full((t, 1), 3, dtype=torch.int32, device=DEV)
        x = randn(gen(t), t, 24, dtype=BF16)
        plan = moe.Dispatch(t, 1, 4, 24).dispatch(ids, x)
        assert plan.offsets.tolist() == [0, 0, 0, 0, t] and torch.equal(plan.x, x)
        plan.dispatch(ids + 4, x)
        assert plan.offsets.tolist() == [0] * 5
        assert bool((plan.slots == -1).all()) and bool((plan.rows == -1).all())
        ids[:] = -(1 << 31)
        assert plan.dispatch(ids, x).offsets.tolist() == [0] * 5


# ---------------------------------------------------------------- combine
COMBINE = [
    # tokens, k, features, rows of y
    (1, 1, 1, 1), (1, 8, 7168, 8), (5, 2, 100, 10), (33, 6, 264, 100), (64, 1, 4104, 64), (7, 32, 72, 200),
    (200, 9, 2049, 500), (3, 4, 8, 0),
]


def some_rows(g, t, k, n):
    """Distinct rows of y in random order, with some choices left out."""
    perm = torch.full((max(t * k, n),), -1, dtype=torch.int32, device=DEV)
    perm[:n] = torch.randperm(n, generator=g, device=DEV, dtype=torch.int32) if n else perm[:n]
    perm = perm[:t * k].reshape(t, k).clone()
    perm[torch.rand(t, k, generator=g, device=DEV) < 0.2] = -1
    if t > 2:
        perm[1] = -1
    return perm


@pytest.mark.parametrize("t,k,h,n", COMBINE)
@pytest.mark.parametrize("dtype,pad,lead", [(BF16, 0, 0), (F32, 0, 0), (BF16, 5, 1), (F32, 4, 4)])
@pytest.mark.parametrize("weighted", [True, False])
def test_combine_and_gradient(t, k, h, n, dtype, pad, lead, weighted):
    g = gen(t * k + h)
    y = strided(randn(g, n, h, dtype=dtype), pad, lead)
    rows = some_rows(g, t, k, n)
    w = randn(g, t, k) if weighted else None
    res = strided(randn(g, t, h, dtype=dtype), pad, lead)
    ok = (rows >= 0)[..., None]
    at = rows.clamp(min=0).long()
    yy = torch.where(ok, y.double()[at], 0.0) if n else torch.zeros(t, k, h, dtype=torch.float64, device=DEV)
    terms = yy * (w.double()[..., None] if weighted else 1.0)
    err = (k + 2) * ref.EPS * (terms.abs().sum(1) + res.double().abs())
    ref.close(moe.combine(y, rows, w), terms.sum(1), err, dtype)
    out = strided(torch.zeros(t, h, dtype=dtype, device=DEV), pad, lead)
    ref.close(moe.combine(y, rows, w, residual=res, out=out), terms.sum(1) + res.double(), err, dtype)
    moe.combine(y, rows, w, residual=res, out=res)  # in place
    assert torch.equal(res, out)

    dout = strided(randn(g, t, h, dtype=dtype), pad, lead)
    dy = torch.full((n, h), 5.0, dtype=dtype, device=DEV)
    _, dw = moe.combine_grad(dout, y, rows, w, dy=dy)
    want = torch.full((n, h), 5.0, dtype=dtype, device=DEV)
    f = (w if weighted else torch.ones(t, k, device=DEV))[..., None] * dout.float()[:, None]  # one rounding each
    keep = rows >= 0
    want[rows[keep].long()] = f[keep].to(dtype)
    assert torch.equal(dy, want)
    if weighted:
        prod = dout.double()[:, None] * yy
        ref.close(dw, prod.sum(2), (h + 2) * ref.EPS * prod.abs().sum(2), F32)


def test_combine_leaves_out_rows_past_the_end_and_zero_weights_follow_ieee():
    y = torch.ones(4, 16, device=DEV)
    y[1] = math.inf
    rows = torch.tensor([[0, 4], [1 << 30, -7], [1, 2]], dtype=torch.int32, device=DEV)
    w = torch.tensor([[2.0, 1.0], [1.0, 1.0], [0.0, 1.0]], device=DEV)
    got = moe.combine(y, rows, w)
    assert bool((got[0] == 2).all()) and bool((got[1] == 0).all()) and bool(torch.isnan(got[2]).all())
    dy = torch.zeros_like(y)
    _, dw = moe.combine_grad(torch.ones(3, 16, device=DEV), y, rows, w, dy=dy)
    assert dw.tolist() == [[16.0, 0.0], [0.0, 0.0], [math.inf, 16.0]]
    assert bool((dy[0] == 2).all()) and bool((dy[3] == 0).all())


def test_rows_past_32_bit_offsets():
    """Rows more than 4 GiB into their matrix."""
    n, h = (1 << 32) // 8192 + 40, 8192  # bfloat16 rows of 16 KiB: past 8 GiB, and past 2^32 elements
    y = torch.zeros(n, h, dtype=BF16, device=DEV)
    y[-3:] = randn(gen(1), 3, h, dtype=BF16)
    rows = torch.tensor([[n - 1, 0], [n - 3, n - 2]], dtype=torch.int32, device=DEV)
    got = moe.combine(y, rows)
    assert torch.equal(got[0], y[-1]) and torch.equal(got[1], (y[-3].float() + y[-2].float()).to(BF16))
    dout = randn(gen(2), 2, h, dtype=BF16)
    dy = torch.zeros_like(y)
    moe.combine_grad(dout, y, rows, dy=dy)
    assert torch.equal(dy[-1], dout[0]) and torch.equal(dy[-2], dout[1]) and torch.equal(dy[-3], dout[1])


# ---------------------------------------------------------------- streams and graphs
def test_on_another_stream_and_in_a_graph():
    t, k, e, h = 300, 4, 16, 128
    g = gen(9)
    logits, x = randn(g, t, e), randn(g, t, h, dtype=BF16)
    plan = moe.Dispatch(t, k, e, h)
    out = torch.empty(t, h, dtype=BF16, device=DEV)
    ids = torch.empty(t, k, dtype=torch.int32, device=DEV)
    w = torch.empty(t, k, device=DEV)

    def layer(stream=None):
        moe.route(logits, k, normalise=True, ids=ids, weights=w, stream=stream)
        plan.dispatch(ids, x, stream=stream)
        moe.combine(plan.x, plan.rows, w, out=out, stream=stream)

    layer()
    torch.cuda.synchronize()
    want = out.clone()
    side = torch.cuda.Stream()
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    layer(side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer()
    for seed in range(3):
        logits.copy_(randn(gen(20 + seed), t, e))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        layer()
        torch.cuda.synchronize()
        assert torch.equal(out, got)


def test_errors_are_raised():
    x = torch.zeros(4, 8, device=DEV)
    with pytest.raises(ll.LLError) as e:
        moe.route(x.half(), 2)
    assert e.value.status == ll.LL_ERR_UNSUPPORTED
    with pytest.raises(ll.LLError):
        moe.route(x, 9)
    with pytest.raises(ValueError):
        moe.route(x.t(), 2)  # no unit stride
    with pytest.raises(ValueError):
        moe.route(x, 2, bias=torch.zeros(7, device=DEV))
    with pytest.raises(ValueError):
        moe.Dispatch(3, 2, 4, 8, F32).dispatch(torch.zeros(4, 2, dtype=torch.int32, device=DEV), x)
    with pytest.raises(ValueError):
        moe.combine(x, torch.zeros(2, 2, dtype=torch.int64, device=DEV))


# ---------------------------------------------------------------- routing of many tokens
# More than 4096 tokens of up to 256 experts and 16 choices take 16 lanes a
# token; one size for each number of logits a lane can hold, and one that does
# not fit them.
ROUTE_MANY = [(4097, 5, 2), (4098, 20, 3), (5003, 60, 8), (4099, 90, 6), (4100, 128, 8), (4097, 160, 6),
              (4101, 190, 16), (4099, 256, 16), (4097, 8, 8), (4111, 16, 1), (4097, 257, 4), (4097, 40, 17)]


def choose(logits, bias, k):
    """The k largest binary32 keys a row, ties to the lowest index, on the CPU."""
    key = (logits.float() if bias is None else logits.float() + bias).cpu()
    key = torch.where(torch.isnan(key), torch.full_like(key, -math.inf), key)
    val, idx = torch.sort(key, dim=1, descending=True, stable=True)
    return torch.where(val[:, :k] > -math.inf, idx[:, :k], -1).to(logits.device)


def check_route(t, e, k, dtype, score, normalise, biased, masked, pad):
    x = route_inputs(t, e, dtype, t + e, masked)
    bias = 0.3 * randn(gen(e), e) if biased else None
    v = strided(x, pad)
    ids, w = moe.route(v, k, bias=bias, score=score, normalise=normalise, scale=2.5)
    want_ids = choose(x, bias, k)
    assert torch.equal(ids.long(), want_ids)
    rel = (e + k + 48) * ref.EPS  # as in test_route_and_gradient
    want_w = route_weights64(x.double(), want_ids, score, normalise, 2.5)
    ref.close(w, want_w, want_w.abs() * rel, F32)
    g = randn(gen(3), t, k)
    got = moe.route_grad(v, ids, g, score=score, normalise=normalise, scale=2.5)
    want = route_grad64(x.double(), want_ids, g.double(), score, normalise, 2.5)
    size = 2.5 * (g.abs() * (want_ids >= 0)).sum(1, keepdim=True).double()
    ref.close(got, want, size * rel * torch.ones_like(want), dtype)


@pytest.mark.parametrize("t,e,k", ROUTE_MANY)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("score,normalise,biased,masked,pad", [
    ("softmax", False, False, True, 0), ("softmax", False, True, True, 3), ("softmax", True, True, False, 0),
    ("sigmoid", False, False, True, 1), ("sigmoid", True, True, False, 8)])
def test_route_of_many_tokens(t, e, k, dtype, score, normalise, biased, masked, pad):
    check_route(t, e, k, dtype, score, normalise, biased, masked, pad)


@pytest.mark.parametrize("t,e,k", [(1, 8, 8), (33, 64, 8), (7, 257, 4), (3, 1000, 32), (130, 160, 6)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("score,masked,pad", [("softmax", False, 0), ("softmax", True, 3), ("sigmoid", True, 0)])
def test_biased_route_without_normalisation(t, e, k, dtype, score, masked, pad):
    """Keys have the bias; the softmax is that of the logits alone."""
    check_route(t, e, k, dtype, score, False, True, masked, pad)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_ties_of_many_tokens_go_to_the_lowest_index(dtype):
    t = 5000
    for e in (16, 60, 256):
        x = torch.zeros(t, e, device=DEV)
        x[1::5, e // 2:] = 1.0
        x[2::5] = -0.0
        x[2::5, 3] = 0.0  # equal to -0
        x[3::5, 1::2] = -math.inf
        x[4::5] = math.inf
        want = torch.zeros(t, 4, dtype=torch.int32)
        for r, row in enumerate(([0, 1, 2, 3], [e // 2 + i for i in range(4)], [0, 1, 2, 3], [0, 2, 4, 6],
                                 [0, 1, 2, 3])):
            want[r::5] = torch.tensor(row, dtype=torch.int32)
        ids, _ = moe.route(x.to(dtype), 4)
        assert torch.equal(ids.cpu(), want)
        ids, _ = moe.route(x.to(dtype), 4, bias=torch.zeros(e, device=DEV))
        assert torch.equal(ids.cpu(), want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("normalise", [False, True])
def test_sigmoid_gradient_keeps_its_relative_accuracy(normalise, dtype):
    """1 - sigmoid(x) of a large x is a small value like any other, not the
    rounding error of a subtraction.  A few exponentials, sums of two positive
    terms and quotients, each good to a few units."""
    x = torch.linspace(-30, 60, 400).to(dtype).to(DEV)[:, None].repeat(1, 3)
    x[:, 1] -= 1.0
    x[:, 2] = -math.inf
    g = torch.zeros(400, 2, device=DEV)
    g[:, 0] = 1.0
    ids = torch.tensor([[0, 1]], dtype=torch.int32, device=DEV).repeat(400, 1)
    got = moe.route_grad(x, ids, g, score="sigmoid", normalise=normalise)
    l = x.double()
    p, q = torch.sigmoid(l), torch.sigmoid(-l)
    want = torch.zeros(400, 3, dtype=torch.float64, device=DEV)
    if normalise:  # u (g - sum u g) (1 - p), and g - sum u g = 1 - u0 = u1
        u0 = p[:, 0] / (p[:, 0] + p[:, 1])
        u1 = p[:, 1] / (p[:, 0] + p[:, 1])
        want[:, 0], want[:, 1] = u0 * u1 * q[:, 0], -u1 * u0 * q[:, 1]
    else:
        want[:, 0] = p[:, 0] * q[:, 0]
    ref.close(got, want, want.abs() * 64 * ref.EPS, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("top", [-60.0, -95.0, -300.0, -600.0])
@pytest.mark.parametrize("tokens", [9, 4200])
def test_normalised_sigmoid_of_small_scores(top, dtype, tokens):
    """Scores below binary32's range still have their shares of the sum; those
    below binary64's, as of masks of the type's lowest value, have none."""
    e, k = 20, 5
    x = (top - 12 * torch.rand(tokens, e, generator=gen(7), device=DEV)).to(dtype)
    x[1::3, ::2] = torch.finfo(dtype).min
    x[2::3] = torch.finfo(dtype).min
    ids, w = moe.route(x, k, score="sigmoid", normalise=True, scale=2.5)
    want_ids = choose(x, None, k)
    assert torch.equal(ids.long(), want_ids)
    want = route_weights64(x.double(), want_ids, "sigmoid", True, 2.5)
    # differences of logits below 16 rounded once, and the exponentials' few units of them
    rel = (k + 48 + 16) * ref.EPS
    ref.close(w, want, want.abs() * rel, F32)
    assert bool((w[2::3] == 0).all()) and bool((w[::3].sum(1) > 2.4).all())
    g = randn(gen(8), tokens, k)
    got = moe.route_grad(x, ids, g, score="sigmoid", normalise=True, scale=2.5)
    p = torch.sigmoid(x.double())
    u = want / 2.5
    gg = 2.5 * g.double()
    c = u * (gg - (u * gg).sum(1, keepdim=True)) * (1 - p.gather(1, want_ids))
    full = torch.zeros(tokens, e, dtype=torch.float64, device=DEV).scatter_(1, want_ids, c)
    size = 2.5 * g.abs().sum(1, keepdim=True).double()
    ref.close(got, full, size * rel * torch.ones_like(full), dtype)


def test_weight_gradient_of_an_unweighted_combine():
    """Asked for by giving its memory; weights of 1 have a gradient too."""
    g = gen(27)
    y, dout = randn(g, 12, 40), randn(g, 5, 40)
    rows = some_rows(g, 5, 2, 10)
    dw = torch.full((5, 2), math.nan, device=DEV)
    dy, got = moe.combine_grad(dout, y, rows, dweights=dw)
    assert got is dw
    prod = dout.double()[:, None] * torch.where((rows >= 0)[..., None], y.double()[rows.clamp(min=0).long()], 0.0)
    ref.close(dw, prod.sum(2), 42 * ref.EPS * prod.abs().sum(2), F32)
    assert torch.equal(dy, moe.combine_grad(dout, y, rows, torch.ones(5, 2, device=DEV))[0])
    assert moe.combine_grad(dout, y, rows)[1] is None


def test_combine_and_gradient_of_rows_without_features():
    y, rows = torch.zeros(4, 0, device=DEV), torch.tensor([[0, 1], [2, -1]], dtype=torch.int32, device=DEV)
    assert moe.combine(y, rows).shape == (2, 0)
    dy, dw = moe.combine_grad(torch.zeros(2, 0, device=DEV), y, rows, torch.ones(2, 2, device=DEV),
                              dweights=torch.full((2, 2), math.nan, device=DEV))
    assert dy.shape == (4, 0) and dw.tolist() == [[0.0, 0.0], [0.0, 0.0]]


def test_a_refused_dispatch_leaves_the_plan_as_it_was():
    ids = torch.randint(0, 8, (6, 2), generator=gen(28), device=DEV, dtype=torch.int32)
    x = randn(gen(29), 6, 16)
    plan = moe.Dispatch(10, 2, 8, 16, F32).dispatch(ids, x)
    kept = plan.rows.clone()
    for bad_ids, bad_x in ((ids[:4], x), (ids[:4].long(), x[:4]), (ids[:4], x[:4].bfloat16())):
        with pytest.raises(ValueError):
            plan.dispatch(bad_ids, bad_x)
        assert plan.tokens == 6 and plan.rows.shape == (6, 2) and plan.x.shape == (12, 16)
        assert torch.equal(plan.rows, kept)
    assert plan.dispatch(ids[:4], x[:4]).tokens == 4


@pytest.mark.parametrize("tokens", [1, 300, 4200])
@pytest.mark.parametrize("normalise", [False, True])
def test_a_selection_bias_on_the_scores(tokens, normalise):
    """The way route's documentation gives: choice by score + bias, weights and
    gradient of the scores alone."""
    e, k, scale = 64, 6, 2.5
    logits = 2 * randn(gen(50), tokens, e)
    bias = 0.2 * randn(gen(51), e)
    scores = torch.sigmoid(logits)
    ids, _ = moe.route(scores, k, bias=bias)
    assert torch.equal(ids.long(), choose(scores, bias, k))
    if tokens > 1:  # not what the same bias on the logits chooses
        assert not torch.equal(ids, moe.route(logits, k, bias=bias, score="sigmoid")[0])
    w = scores.gather(1, ids.long())
    if normalise:
        w = w / w.sum(1, keepdim=True)
    want = route_weights64(logits.double(), ids.long(), "sigmoid", normalise, 1.0)
    rel = (e + k + 48) * ref.EPS
    ref.close(w, want, want * rel, F32)
    g = randn(gen(52), tokens, k)
    got = moe.route_grad(logits, ids, g, score="sigmoid", normalise=normalise, scale=scale)
    want = route_grad64(logits.double(), ids.long(), g.double(), "sigmoid", normalise, scale)
    ref.close(got, want, scale * g.abs().sum(1, keepdim=True).double() * rel * torch.ones_like(want), F32)
