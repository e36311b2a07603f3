"""The expert-layer C ABI on the CPU: what include/llmoe.h declares is exported
and bound, and bad arguments are refused before any HIP call (no GPU needed)."""
from __future__ import annotations

import os
import re

import pytest

from paper_2607_16100_amd import llcoll as ll
from paper_2607_16100_amd import llmoe as lm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = ll.LL_F32, ll.LL_BF16
# fake device addresses, far apart: never dereferenced
A, B, C, D, E, F = (k << 40 for k in range(1, 7))


def test_header_and_binding_agree():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "llmoe.h")).read(), flags=re.S)
    names = set(re.findall(r"^int (ll_[a-z_0-9]+)\s*\(", text, flags=re.M))
    assert names == set(lm.exported_symbols())
    for n in names:
        assert hasattr(ll.library(), n), n
    for name, value in re.findall(r"(LL_(?:ACT|SCORE|LINEAR)_[A-Z_]+) = (\d+)", text):
        assert getattr(lm, name) == int(value), name
    for name, value in re.findall(r"#define (LL_(?:GRAD|MOE)_[A-Z0-9_]+) (\w+)", text):
        assert getattr(lm, name) == int(value.rstrip("u"), 0), name


def route(logits=A, ld=64, tokens=4, experts=64, k=4, dt=F32, bias=0, score=0, ids=B, weights=C):
    return lm.ll_moe_route(logits, ld, tokens, experts, k, dt, bias, score, 0, 1.0, ids, weights, 0)


def route_grad(logits=A, ld=64, tokens=4, experts=64, k=4, dt=F32, score=0, ids=B, dweights=C, dlogits=D, ldd=64):
    return lm.ll_moe_route_grad(logits, ld, tokens, experts, k, dt, score, 0, 1.0, ids, dweights, dlogits, ldd, 0)


@pytest.mark.parametrize("kw,want", [
    (dict(logits=0), ll.LL_ERR_INVALID), (dict(ids=0), ll.LL_ERR_INVALID), (dict(logits=A + 2), ll.LL_ERR_INVALID),
    (dict(ld=63), ll.LL_ERR_INVALID), (dict(k=0), ll.LL_ERR_INVALID), (dict(k=33), ll.LL_ERR_INVALID),
    (dict(k=8, experts=7), ll.LL_ERR_INVALID), (dict(score=2), ll.LL_ERR_INVALID),
    (dict(experts=0), ll.LL_ERR_INVALID), (dict(experts=1025, ld=1025), ll.LL_ERR_UNSUPPORTED),
    (dict(dt=2), ll.LL_ERR_UNSUPPORTED), (dict(tokens=1 << 24), ll.LL_ERR_UNSUPPORTED),
    (dict(tokens=0), ll.LL_OK),
])
def test_route_refusals(kw, want):
    assert route(**kw) == want
    assert route_grad(**kw) == want


def test_route_refusals_of_one_side():
    assert route(weights=0) == ll.LL_ERR_INVALID
    assert route(bias=A + 2) == ll.LL_ERR_INVALID
    assert route_grad(dweights=0) == ll.LL_ERR_INVALID
    assert route_grad(dlogits=0) == ll.LL_ERR_INVALID
    assert route_grad(ldd=60) == ll.LL_ERR_INVALID
    assert route_grad(dlogits=A + 256) == ll.LL_ERR_INVALID  # overlaps the logits


def dispatch(ids=A, tokens=4, k=2, first=0, experts=8, x=B, ldx=64, features=64, dt=BF16, offsets=C, slots=C + 4096,
             rows=C + 8192, y=D, ldy=64, ws=0, ws_bytes=0):
    return lm.ll_moe_dispatch(ids, tokens, k, first, experts, x, ldx, features, dt, offsets, slots, rows, y, ldy, ws,
                              ws_bytes, 0)


@pytest.mark.parametrize("kw,want", [
    (dict(ids=0), ll.LL_ERR_INVALID), (dict(offsets=0), ll.LL_ERR_INVALID), (dict(slots=0), ll.LL_ERR_INVALID),
    (dict(rows=0), ll.LL_ERR_INVALID), (dict(y=0), ll.LL_ERR_INVALID), (dict(x=0), ll.LL_ERR_INVALID),
    (dict(first=-1), ll.LL_ERR_INVALID), (dict(k=0), ll.LL_ERR_INVALID), (dict(experts=0), ll.LL_ERR_INVALID),
    (dict(experts=2000), ll.LL_ERR_UNSUPPORTED), (dict(dt=5), ll.LL_ERR_UNSUPPORTED),
    (dict(ldx=63), ll.LL_ERR_INVALID), (dict(ldy=63), ll.LL_ERR_INVALID), (dict(x=B + 1), ll.LL_ERR_INVALID),
    (dict(y=B + 128), ll.LL_ERR_INVALID),
    (dict(tokens=5000), ll.LL_ERR_INVALID),                          # needs a workspace
    (dict(tokens=5000, ws=E, ws_bytes=16), ll.LL_ERR_SCRATCH),
    (dict(tokens=1 << 26, k=32), ll.LL_ERR_UNSUPPORTED),
])
def test_dispatch_refusals(kw, want):
    assert dispatch(**kw) == want


def test_dispatch_workspace_size():
    assert lm.ll_moe_dispatch_bytes(16, 8, 256) == (ll.LL_OK, 0)
    st, n = lm.ll_moe_dispatch_bytes(8192, 8, 256)
    assert st == ll.LL_OK and 0 < n <= 128 * 256 * 4
    for tokens in (129, 1000, 4097, 65537, 1 << 20, (1 << 24) - 1):
        st, n = lm.ll_moe_dispatch_bytes(tokens, 8, 1024)
        assert st == ll.LL_OK and 0 < n <= 128 * 1024 * 4
    assert lm.ll_moe_dispatch_bytes(16, 8, 0)[0] == ll.LL_ERR_INVALID


def combine(y=A, ldy=64, nrows=8, rows=B, weights=C, residual=0, ldr=64, tokens=4, k=2, features=64, dt=BF16, out=D,
            ldo=64):
    return lm.ll_moe_combine(y, ldy, nrows, rows, weights, residual, ldr, tokens, k, features, dt, out, ldo, 0)


def combine_grad(dout=E, ldd=64, y=A, ldy=64, nrows=8, rows=B, weights=C, tokens=4, k=2, features=64, dt=BF16, dy=D,
                 lddy=64, dweights=F):
    return lm.ll_moe_combine_grad(dout, ldd, y, ldy, nrows, rows, weights, tokens, k, features, dt, dy, lddy,
                                  dweights, 0)


@pytest.mark.parametrize("kw,want", [
    (dict(y=0), ll.LL_ERR_INVALID), (dict(rows=0), ll.LL_ERR_INVALID), (dict(k=0), ll.LL_ERR_INVALID),
    (dict(ldy=63), ll.LL_ERR_INVALID), (dict(dt=7), ll.LL_ERR_UNSUPPORTED), (dict(y=A + 1), ll.LL_ERR_INVALID),
    (dict(tokens=0), ll.LL_OK), (dict(nrows=1 << 31), ll.LL_ERR_UNSUPPORTED),
])
def test_combine_refusals(kw, want):
    assert combine(**kw) == want
    assert combine_grad(**kw) == want


def test_combine_refusals_of_one_side():
    assert combine(out=0) == ll.LL_ERR_INVALID
    assert combine(out=A + 64) == ll.LL_ERR_INVALID
    assert combine(residual=D + 32) == ll.LL_ERR_INVALID  # overlaps the output without being it
    assert combine(residual=E, ldr=60) == ll.LL_ERR_INVALID
    assert combine_grad(dout=0) == ll.LL_ERR_INVALID
    assert combine_grad(dy=0) == ll.LL_ERR_INVALID
    assert combine_grad(dy=A) == ll.LL_ERR_INVALID
    assert combine_grad(dy=E + 2) == ll.LL_ERR_INVALID


def d(rows=8, in_=64, out=32, act=0, groups=1, dt=BF16, **fields):
    return lm.desc(dt, act, groups, rows, in_, out, **fields)


def test_desc_init():
    x = lm.desc(BF16, lm.LL_ACT_SWIGLU, 4, 100, 64, 32)
    assert (x.groups, x.rows, x.in_, x.out, x.ldx, x.ldw, x.wstride, x.ldy, x.ldz, x.ldr) == (
        4, 100, 64, 32, 64, 64, 2048, 16, 32, 16)
    assert ll.library().ll_linear_desc_init(None, 0, 0, 1, 1, 1, 1) == ll.LL_ERR_INVALID


def three(desc, p=A, q=B, out=C):
    """The three products with the same descriptor (no activation)."""
    return (lm.ll_linear(desc, p, q, 0, 0, out, 0, 0, 0, 0), lm.ll_linear_grad_x(desc, p, q, 0, out, 0, 0, 0),
            lm.ll_linear_grad_w(desc, p, q, out, 0, 0, 0, 0, 0))


@pytest.mark.parametrize("kw,want", [
    (dict(size=4), ll.LL_ERR_INVALID), (dict(groups=0), ll.LL_ERR_INVALID), (dict(groups=2), ll.LL_ERR_INVALID),
    (dict(groups=2000, offsets=E), ll.LL_ERR_UNSUPPORTED), (dict(dt=3), ll.LL_ERR_UNSUPPORTED),
    (dict(act=9), ll.LL_ERR_INVALID), (dict(in_=0), ll.LL_ERR_INVALID), (dict(out=0), ll.LL_ERR_INVALID),
    (dict(ldw=63), ll.LL_ERR_INVALID), (dict(groups=2, offsets=E, wstride=100), ll.LL_ERR_INVALID),
    (dict(offsets=E + 2), ll.LL_ERR_INVALID), (dict(rows=1 << 31), ll.LL_ERR_UNSUPPORTED),
    (dict(in_=(1 << 20) + 1), ll.LL_ERR_UNSUPPORTED), (dict(ldy=31), ll.LL_ERR_INVALID),
    (dict(ldx=63), ll.LL_ERR_INVALID),
])
def test_linear_refusals(kw, want):
    assert three(d(**kw)) == (want,) * 3


def test_linear_refusals_of_pointers():
    x = d()
    bad = (ll.LL_ERR_INVALID,) * 3
    assert three(x, p=0) == bad and three(x, q=0) == bad and three(x, out=0) == bad
    assert three(x, p=A + 1) == bad and three(x, out=C + 1) == bad
    assert three(x, out=A + 16) == bad  # overlaps an input
    assert lm.ll_linear(d(act=lm.LL_ACT_SWIGLU, out=33), A, B, 0, 0, C, 0, 0, 0, 0) == ll.LL_ERR_INVALID
    assert lm.ll_linear(x, A, B, 0, C + 64, C, 0, 0, 0, 0) == ll.LL_ERR_INVALID  # residual overlaps y
    assert lm.ll_linear(x, A, B, 0, 0, C, C + 8, 0, 0, 0) == ll.LL_ERR_INVALID   # z overlaps y
    assert lm.ll_linear(x, A, B, E + 1, 0, C, 0, 0, 0, 0) == ll.LL_ERR_INVALID   # misaligned bias
    assert lm.ll_linear(x, A, B, 0, 0, C, 0, E + 8, 64, 0) == ll.LL_ERR_INVALID  # misaligned workspace
    assert lm.ll_linear_grad_x(d(act=lm.LL_ACT_GELU), A, B, 0, C, 0, 0, 0) == ll.LL_ERR_INVALID  # no z
    assert lm.ll_linear_grad_x(d(act=lm.LL_ACT_SWIGLU, ldy=32, ldz=128), A, B, E, C, 0, 0, 0) == ll.LL_ERR_INVALID
    assert lm.ll_linear_grad_w(x, A, B, C, 0, 8, 0, 0, 0) == ll.LL_ERR_INVALID   # unknown flag
    assert lm.ll_linear_grad_w(x, A, B, C, C + 64, 0, 0, 0, 0) == ll.LL_ERR_INVALID
    # binary32 gradients need binary32 alignment
    assert lm.ll_linear_grad_w(x, A, B, C + 2, 0, lm.LL_GRAD_F32, 0, 0, 0) == ll.LL_ERR_INVALID


def test_linear_without_rows_launches_nothing():
    assert lm.ll_linear(d(rows=0), 0, 0, 0, 0, 0, 0, 0, 0, 0) == ll.LL_OK
    assert lm.ll_linear_grad_x(d(rows=0), 0, 0, 0, 0, 0, 0, 0) == ll.LL_OK


def test_linear_bytes():
    assert lm.ll_linear_bytes(d(), 3)[0] == ll.LL_ERR_INVALID
    assert lm.ll_linear_bytes(d(size=3), 0)[0] == ll.LL_ERR_INVALID
    for which in range(3):
        assert lm.ll_linear_bytes(d(), which)[0] == ll.LL_OK


def act_grad(dy=A, z=B, rows=4, features=8, dt=F32, act=lm.LL_ACT_SILU, dz=C, lddy=8, ldz=16, lddz=16):
    return lm.ll_act_grad(dy, lddy, z, ldz, rows, features, dt, act, dz, lddz, 0)


def test_act_grad_refusals():
    assert act_grad(dy=0) == act_grad(z=0) == act_grad(dz=0) == ll.LL_ERR_INVALID
    assert act_grad(act=6) == act_grad(lddy=7) == ll.LL_ERR_INVALID
    assert act_grad(act=lm.LL_ACT_SWIGLU, ldz=15) == ll.LL_ERR_INVALID
    assert act_grad(dz=A + 4) == ll.LL_ERR_INVALID
    assert act_grad(dt=4) == ll.LL_ERR_UNSUPPORTED
    assert act_grad(rows=0) == ll.LL_OK


def test_extents_of_zero():
    assert route(tokens=0, logits=0, ids=0, weights=0) == ll.LL_OK
    assert route_grad(tokens=0, logits=0, ids=0, dweights=0, dlogits=0) == ll.LL_OK
    assert combine(tokens=0, y=0, rows=0, out=0) == combine_grad(tokens=0, dout=0, rows=0) == ll.LL_OK
    assert dispatch(tokens=0, offsets=0) == ll.LL_ERR_INVALID  # offsets are written all the same


def test_act_grad_of_nothing():
    for act, wide in ((lm.LL_ACT_SILU, 8), (lm.LL_ACT_SWIGLU, 16)):
        assert act_grad(dy=0, z=0, dz=0, rows=0, act=act, ldz=wide, lddz=wide) == ll.LL_OK
        assert act_grad(dy=0, z=0, dz=0, features=0, act=act) == ll.LL_OK
        assert act_grad(dy=0, rows=1, act=act) == ll.LL_ERR_INVALID


def test_combine_gradient_without_features_needs_no_rows():
    assert combine_grad(features=0, dout=0, y=0, dy=0, dweights=0) == ll.LL_OK
    assert combine_grad(features=0, dout=0, y=0, dy=0, rows=0) == ll.LL_ERR_INVALID
    assert combine(features=0, y=0, out=0, rows=0) == ll.LL_OK


@pytest.mark.parametrize("kw", [
    dict(rows=A), dict(slots=A + 16), dict(offsets=A + 28), dict(slots=C + 32), dict(rows=C + 4096 + 28),
    dict(y=C + 8192), dict(slots=D + 128), dict(x=C + 16), dict(offsets=B + 4),
    # 40000 bytes of ids, slots and rows each, and a workspace
    dict(tokens=5000, slots=E, rows=F, ws=A + 39996, ws_bytes=1 << 20),
    dict(tokens=5000, slots=E, rows=F, ws=C + 32, ws_bytes=1 << 20),
    dict(tokens=5000, slots=E, rows=E + 39996, ws=F, ws_bytes=1 << 20),
])
def test_dispatch_refuses_outputs_over_its_other_arrays(kw):
    """Places come from ids that are read twice, and rows of y from places: an
    output over them would send rows anywhere."""
    assert dispatch(**kw) == ll.LL_ERR_INVALID


def test_rows_without_features_overlap_nothing():
    assert combine_grad(features=0, dout=A, y=A, dy=A, dweights=0) == ll.LL_OK


def test_limits_of_a_products_weight():
    """No rows: nothing is launched, but the shape is checked.  128256 x 16384 bfloat16 is 4.2 GB."""
    for dt, in_ in ((BF16, 16384), (F32, 8192)):
        big = dict(rows=0, in_=in_, out=128256, dt=dt)
        assert lm.ll_linear(d(**big), 0, 0, 0, 0, 0, 0, 0, 0, 0) == ll.LL_OK
        assert lm.ll_linear_grad_x(d(**big), 0, 0, 0, 0, 0, 0, 0) == ll.LL_OK
        for which in range(3):
            assert lm.ll_linear_bytes(d(**big), which)[0] == ll.LL_OK
        gated = d(act=lm.LL_ACT_SWIGLU, **big)
        assert lm.ll_linear(gated, 0, 0, 0, 0, 0, 0, 0, 0, 0) == ll.LL_ERR_UNSUPPORTED
        assert [lm.ll_linear_bytes(gated, which)[0] for which in range(3)] == [ll.LL_ERR_UNSUPPORTED, ll.LL_OK, ll.LL_OK]
    for ld in ("ldx", "ldw", "ldy"):
        assert three(d(**{ld: 1 << 21}, rows=0))[:2] == (ll.LL_OK,) * 2
        assert three(d(**{ld: (1 << 21) + 1}, rows=0)) == (ll.LL_ERR_UNSUPPORTED,) * 3
