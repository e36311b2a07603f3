"""Norms around a block and their gradients on the GPU against plain 64-bit
forms, the gradients against differences as well."""
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
LAYOUTS = [(0, 0), (3, 1), (8, 0)]

# tokens, features: a wave a row, 128 to 1024 threads with one chunk, 1024 with two; ends inside them
SHAPES = [(1, 1), (3, 7), (5, 128), (37, 200), (9, 512), (6, 513), (2100, 1024), (7, 1030), (11, 2048), (600, 2056),
          (4, 4100), (1200, 4096), (530, 5000), (513, 8192), (2, 7168), (3, 8193), (300, 12288), (5, 16384)]
# post, gate, residual, scale, weight
FORMS = [(True, True, True, 0.5, True), (False, False, True, 1.0, True), (False, False, False, 1.0, True),
         (True, False, False, 1.0, True), (False, True, True, -2.0, True), (True, True, True, 0.25, False)]


def d(t):
    return None if t is None else t.double()


def inputs(n, f, dtype, form, layout, wdt=None, seed=0):
    post, gate, residual, scale, weight = form
    g = gen(n + f + seed)
    wdt = wdt or dtype
    s = {"y": strided(randn(g, n, f, dtype=dtype) * 1.5, *LAYOUTS[layout]),
         "x": strided(3 * randn(g, n, f, dtype=dtype), *LAYOUTS[layout]) if residual else None,
         "gate": torch.sigmoid(randn(g, n)) if gate else None,
         "post": (1 + 0.3 * randn(g, f)).to(wdt) if post else None,
         "weight": (1 + 0.3 * randn(g, f)).to(wdt) if weight else None, "scale": scale, "g": g}
    return s


@pytest.mark.parametrize("n,f", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("form,layout", [(0, 0), (1, 1), (2, 2), (3, 0), (4, 1), (5, 0)])
def test_norm(n, f, dtype, form, layout):
    eps = 1e-5
    s = inputs(n, f, dtype, FORMS[form], layout, wdt=F32 if form == 3 else None)
    got = moe.norm(s["y"], s["weight"], residual=s["x"], gate=s["gate"], scale=s["scale"], post=s["post"], eps=eps,
                   quantised=s["weight"] is not None and form != 2)
    h, eh, r, er = bref.norm(d(s["y"]), d(s["x"]), d(s["gate"]), s["scale"], d(s["post"]), d(s["weight"]), eps)
    if form == 2:
        assert got.r is None
    else:
        ref.close(got.r, r, er, dtype)
    if s["weight"] is None:
        assert got.h is None and got.q is None
        return
    ref.close(got.h, h, eh, dtype)
    if got.q is not None:
        sc = got.q_scales.view(torch.uint8).long()
        amax = torch.stack([p.abs().amax(1) for p in h.split(128, 1)], 1)
        slack = torch.stack([p.amax(1) for p in eh.split(128, 1)], 1)
        assert bool(((sc >= bref.exponents((amax - slack).clamp(min=0))) & (sc <= bref.exponents(amax + slack))).all())
        step = bref.stretch(sc, f, 1)
        bound = (eh + (h.abs() + eh) * 2.0 ** -4).maximum(step * 2.0 ** -10 + eh)
        assert bool(((got.q.double() * step - h).abs() <= bound * 1.0001).all())
        if dtype is F32:  # then h is what was rounded
            q, s2 = moe.quantise(got.h)
            assert torch.equal(q.view(torch.uint8), got.q.view(torch.uint8))
            assert torch.equal(s2.view(torch.uint8), got.q_scales.view(torch.uint8))


@pytest.mark.parametrize("n,f", SHAPES + [(1500, 300), (1, 8192)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("form,layout", [(0, 0), (1, 1), (2, 2), (3, 0), (4, 1), (5, 0)])
def test_gradients(n, f, dtype, form, layout):
    eps = 1e-5
    s = inputs(n, f, dtype, FORMS[form], layout, wdt=F32 if form == 3 else None, seed=1)
    g = s["g"]
    weight = s["weight"]
    r = strided(2 * randn(g, n, f, dtype=dtype), *LAYOUTS[layout]) if weight is not None else None
    dh = strided(randn(g, n, f, dtype=dtype), *LAYOUTS[layout]) if weight is not None else None
    dr = strided(randn(g, n, f, dtype=dtype), *LAYOUTS[layout]) if form not in (2, 3) else None
    y = s["y"] if s["post"] is not None or s["gate"] is not None else None
    got = moe.norm_grad(dh, r, weight, dr=dr, y=y, gate=s["gate"], scale=s["scale"], post=s["post"], eps=eps)
    want = bref.norm_grad(d(dh), d(r), d(dr), d(s["y"]), d(s["gate"]), s["scale"], d(s["post"]), d(weight), eps)
    ref.close(got.dr, *want["dr"], dtype)
    ref.close(got.dy, *want["dy"], dtype)
    assert (got.dy is got.dr) == (form in (1, 2))
    for name in ("dgate", "dweight", "dpost"):
        t = getattr(got, name)
        assert (t is None) == (name not in want)
        if t is not None:
            ref.close(t, *want[name], F32)


@pytest.mark.parametrize("form", range(5))
def test_gradients_against_differences(form):
    """The formulas themselves: central differences of the 64-bit form."""
    n, f, eps = 4, 40, 1e-5
    s = inputs(n, f, F32, FORMS[form], 0, seed=2)
    g = s["g"]
    ch, cr = randn(g, n, f).double(), randn(g, n, f).double()
    names = ["y", "x", "gate", "post", "weight"]

    def value(at):
        h, _, r, _ = bref.norm(at["y"], at["x"], at["gate"], s["scale"], at["post"], at["weight"], eps)
        return float((h * ch).sum() + (r * cr).sum())

    at = {k: d(s[k]) for k in names}
    _, _, r, _ = bref.norm(at["y"], at["x"], at["gate"], s["scale"], at["post"], at["weight"], eps)
    y = s["y"] if s["post"] is not None or s["gate"] is not None else None
    got = moe.norm_grad(ch.float(), r.float(), s["weight"], dr=cr.float(), y=y, gate=s["gate"], scale=s["scale"],
                        post=s["post"], eps=eps)
    grads = {"y": got.dy, "x": got.dr if s["x"] is not None else None, "gate": got.dgate, "post": got.dpost,
             "weight": got.dweight}
    step = 1e-6
    for k in names:
        if at[k] is None:
            continue
        flat, gr = at[k].view(-1), grads[k].reshape(-1).double()
        scale = float(gr.abs().max())
        for i in range(0, flat.numel(), max(1, flat.numel() // 7)):
            keep = float(flat[i])
            flat[i] = keep + step
            up = value(at)
            flat[i] = keep - step
            down = value(at)
            flat[i] = keep
            # differences: 64-bit rounding of a value over the step, the third derivative; gradients: binary32
            assert abs((up - down) / (2 * step) - float(gr[i])) <= 1e-4 * scale + 1e-6 * abs(up)


def test_rows_of_zeros_and_rows_that_are_no_number():
    y = randn(gen(1), 5, 300)
    y[1] = 0
    y[3, 7] = math.nan
    got = moe.norm(y, torch.ones(300, device=DEV), quantised=True)
    assert bool((got.h[1] == 0).all()) and bool((got.q[1].float() == 0).all())
    assert bool(torch.isnan(got.h[3]).all()) and bool(torch.isnan(got.q[3].float()).all())
    assert bool(torch.isfinite(got.h[[0, 1, 2, 4]]).all())


def test_in_place_and_added_gradients():
    g = gen(2)
    n, f = 70, 520
    x, y, w, p = randn(g, n, f), randn(g, n, f), 1 + randn(g, f), 1 + randn(g, f)
    gate = torch.sigmoid(randn(g, n))
    want = moe.norm(y, w, residual=x, gate=gate, post=p, scale=0.5)
    stream = x.clone()
    got = moe.norm(y, w, residual=stream, gate=gate, post=p, scale=0.5, r=stream)
    assert got.r is stream and torch.equal(stream, want.r) and torch.equal(got.h, want.h)
    dh, dr = randn(g, n, f), randn(g, n, f)
    first = moe.norm_grad(dh, want.r, w, dr=dr, y=y, gate=gate, post=p, scale=0.5)
    dw, dp = torch.full((f,), 2.0, device=DEV), torch.full((f,), -3.0, device=DEV)
    dr2, y2 = dr.clone(), y.clone()
    again = moe.norm_grad(dh, want.r, w, dr=dr2, y=y2, gate=gate, post=p, scale=0.5, dr_out=dr2, dy=y2, dweight=dw,
                          dpost=dp, add=True)
    assert torch.equal(again.dr, first.dr) and torch.equal(again.dy, first.dy)
    assert torch.equal(dw, first.dweight + 2) and torch.equal(dp, first.dpost - 3)


def test_no_rows():
    w = torch.ones(40, device=DEV)
    e = torch.zeros(0, 40, device=DEV)
    got = moe.norm(e, w, quantised=True)
    assert got.h.shape == (0, 40) and got.q.shape == (0, 40)
    grads = moe.norm_grad(e, e, w, y=e, post=w, gate=torch.zeros(0, device=DEV))
    assert bool((grads.dweight == 0).all()) and bool((grads.dpost == 0).all()) and grads.dr.shape == (0, 40)
    dw = torch.full((40,), 5.0, device=DEV)
    moe.norm_grad(e, e, w, dweight=dw, add=True)
    assert bool((dw == 5).all())


def test_a_side_stream_and_a_graph():
    g = gen(3)
    n, f = 300, 1032
    y, w, p = randn(g, n, f, dtype=BF16), randn(g, f, dtype=BF16), randn(g, f, dtype=BF16)
    dh, r, gate = randn(g, n, f, dtype=BF16), randn(g, n, f, dtype=BF16), torch.sigmoid(randn(g, n))

    def both(stream=None):
        a = moe.norm(y, w, residual=r, gate=gate, post=p, quantised=True, stream=stream)
        b = moe.norm_grad(dh, r, w, y=y, gate=gate, post=p, stream=stream)
        return [t.view(torch.uint8) if t.element_size() == 1 else t for t in (*a, *b)]

    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        held = both()
    for seed in range(4):
        y.copy_(randn(gen(seed), n, f, dtype=BF16))
        dh.copy_(randn(gen(seed + 9), n, f, dtype=BF16))
        graph.replay()
        torch.cuda.synchronize()
        want = both()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_refusals():
    y, w = torch.zeros(4, 40, device=DEV), torch.ones(40, device=DEV)
    for kw in (dict(weight=None, quantised=True), dict(weight=w.half()), dict(weight=w[:39]),
               dict(weight=w, residual=y.bfloat16()), dict(weight=w, gate=torch.ones(4, dtype=BF16, device=DEV)),
               dict(weight=w, gate=torch.ones(5, device=DEV)), dict(weight=w, post=w.bfloat16()),
               dict(weight=w.clone().requires_grad_()), dict(weight=w, residual=y.clone().requires_grad_()),
               dict(weight=w.cpu())):
        with pytest.raises(ValueError):
            moe.norm(y, **kw)
    for kw in (dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan)):
        with pytest.raises(ll.LLError):
            moe.norm(y, w, **kw)
    with pytest.raises(ll.LLError):
        moe.norm(torch.zeros(1, 16385, device=DEV), torch.ones(16385, device=DEV))
    with pytest.raises(ll.LLError):
        moe.norm(y.half(), w)
    with pytest.raises(ll.LLError):  # h over the residual
        moe.norm(y, w, residual=y.clone(), r=y, h=y)
    for kw in (dict(weight=None), dict(weight=w, post=w), dict(weight=w, gate=torch.ones(4, device=DEV)),
               dict(weight=w, add=True)):
        with pytest.raises(ValueError):
            moe.norm_grad(y, y, **kw)
