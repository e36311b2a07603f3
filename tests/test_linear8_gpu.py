"""Grouped products of 8-bit rows and weights on the GPU against 64-bit forms."""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import blockref as bref  # noqa: E402
import moeref as ref  # noqa: E402
from test_linear_gpu import SHAPES as PLAIN  # noqa: E402
from test_moe_gpu import gen, randn, strided  # noqa: E402

if torch.cuda.is_available():
    from paper_2607_16100_amd import llcoll as ll  # noqa: E402
    from paper_2607_16100_amd import moe  # noqa: E402
else:  # pragma: no cover
    pytest.skip("no GPU", allow_module_level=True)

F32, BF16 = torch.float32, torch.bfloat16
DEV = "cuda"

# rows a group, or None for one group of `rows` without offsets; in, out
SHAPES = dict(PLAIN)
SHAPES.update({
    "blocks": (None, 40, 640, 384),           # five blocks of k
    "eight": ([60, 0, 70], 0, 1024, 320),     # two words of scales
    "split": (None, 48, 7168, 130),           # a long sum of few tiles
    "split_odd": ([50, 41], 0, 2569, 66),     # the same, rows through registers
    "stream": (None, 16, 2176, 96),           # 17 blocks, seven waves of three
    "stream2": ([9, 0, 16, 3], 0, 528, 64),
})


def codes(g, n, k, dtype=torch.uint8):
    """Random finite codes with a normal value's spread, and scales about 1."""
    q = (randn(g, n, k) * torch.exp(randn(g, n, 1)) * 20).clamp(-448, 448).to(moe.E4M3)
    s = torch.randint(120, 130, (n, (k + 127) // 128), generator=g, device=DEV)
    return q, s


def strided8(q, pad, lead):
    """The same codes with rows `pad` further apart, `lead` into their buffer; NaN in between."""
    n, c = q.shape
    buf = torch.full((n * (c + pad) + lead + 16,), 0x7F, dtype=torch.uint8, device=DEV)
    v = buf[lead:lead + n * (c + pad)].view(n, c + pad)[:, :c]
    v.copy_(q.view(torch.uint8))
    return v.view(moe.E4M3)


def case(name, seed):
    counts, rows, i, o = SHAPES[name] if isinstance(name, str) else name
    g = gen(seed)
    if counts is None:
        offsets, n, groups, extra = None, rows, 1, 0
    else:
        extra = 3  # rows that belong to no group
        n, groups = sum(counts) + extra, len(counts)
        offsets = torch.tensor([sum(counts[:c]) for c in range(groups + 1)], dtype=torch.int32, device=DEV)
    xq, xs = codes(g, n, i)
    wq, _ = codes(g, groups * o, i)
    wq = wq.view(groups, o, i)
    ws = torch.randint(118, 126, (groups, (o + 127) // 128, (i + 127) // 128), generator=g, device=DEV)
    return g, n, groups, i, o, offsets, extra, xq, xs, wq, ws


LAYOUTS = [(0, 0), (4, 4), (16, 0), (1, 3)]


def check(name, dtype, act, bias, residual, save, layout, seed=21):
    g, n, groups, i, o, offsets, extra, xq, xs, wq, ws = case(name, seed)
    pad, lead = LAYOUTS[layout]
    x = strided8(xq, pad, lead)
    w = strided8(wq.view(groups * o, i), pad, lead).view(torch.uint8)
    w = w.as_strided((groups, o, i), (o * (i + pad), i + pad, 1)).view(moe.E4M3)
    if extra:
        x[-extra:] = math.nan
    b = randn(g, groups, o, dtype=dtype) if bias else None
    width = o // 2 if act in ref.GATED else o
    rpad, rlead = ((0, 0), (3, 1), (8, 0), (1, 0))[layout]
    res = strided(randn(g, n, width, dtype=dtype), rpad, rlead) if residual else None
    out = torch.full((n, width), 9.0, dtype=dtype, device=DEV)
    z = torch.full((n, o), 9.0, dtype=dtype, device=DEV) if save else None
    sw = bref.wide(ws)
    got = moe.linear8(x, bref.wide(xs), w if offsets is not None else w[0], sw if offsets is not None else sw[0],
                      bias=b, act=act, residual=res, offsets=offsets, out=out, z=z)
    assert got is out
    for gi, lo, hi in ref.spans(offsets, n):
        zz, ez = bref.product8(xq[lo:hi].double(), xs[lo:hi], wq[gi].double(), ws[gi], dtype)
        if bias:
            zz = zz + b[gi].double()
            ez = ez + bref.EPS * zz.abs()
        want, err = ref.act(zz, act), ref.act_err(zz, ez, act)
        if residual:
            want = want + res[lo:hi].double()
            err = err + bref.EPS * want.abs()
        ref.close(out[lo:hi], want, err, dtype)
        if save:
            ref.close(z[lo:hi], zz, ez, dtype)
        if hi - lo > 8 and i >= 64 and dtype is BF16 and act == "none" and not residual:
            # far inside the bound on single values: half a step's root mean square is
            # 2^-9 / sqrt(3) of a value at most, the cut products' about 2^-15
            off = (out[lo:hi].double() - want).norm() / want.norm()
            assert float(off) <= 2.0 ** -9 + 2.0 ** -13
    if extra:
        assert bool((out[-extra:] == 9.0).all()) and (z is None or bool((z[-extra:] == 9.0).all()))


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("act,bias,residual,save,layout", [
    ("none", False, False, False, 0), ("relu", True, False, True, 1), ("gelu", True, True, False, 2),
    ("silu", False, True, True, 3), ("swiglu", True, True, True, 0), ("geglu", False, False, True, 3)])
def test_product(name, dtype, act, bias, residual, save, layout):
    check(name, dtype, act, bias, residual, save, layout)


# 256-wide tiles: whole ones, a short last round in halves ("groups" too), quarters
# and eighths, groups whose last tile has no lower half; 128-wide ones at one and at
# two a CU
LARGE = {
    "full": (None, 4096, 256, 4096),
    "quarters": (None, 4100, 320, 4352),
    "groups": ([700, 0, 130, 2049, 1200, 257], 0, 192, 4104),
    "halves": (None, 4100, 1360, 4880),
    "eighths": (None, 4100, 336, 4096),
    "eighths_groups": ([700, 0, 130, 2049, 1000], 0, 640, 4096),
    "eighths_many": ([40] * 30 + [0] * 40 + [37] * 30 + [1500], 0, 128, 1024),  # more than 64 groups
    "deep": (None, 4096, 1424, 4096),  # twelve stages, the last short
    "odd": (None, 4000, 1408, 4096),   # eleven
    "wide128": (None, 2048, 1664, 2048),
    "many128": (None, 2500, 384, 2048),
}


@pytest.mark.parametrize("name", list(LARGE))
@pytest.mark.parametrize("dtype,act,save,layout", [(BF16, "none", False, 0), (BF16, "swiglu", True, 1),
                                                   (F32, "geglu", False, 0)])
def test_large_products(name, dtype, act, save, layout):
    check(LARGE[name], dtype, act, True, False, save, layout, seed=31)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("layout", [0, 1, 3])
@pytest.mark.parametrize("rows,k,out", [(1, 1, 1), (3, 5, 2), (40, 1, 3), (40, 7, 2), (17, 15, 1), (70, 17, 1), (5, 3, 40),
                                        (66, 129, 65), (66, 143, 3), (66, 257, 3), (66, 385, 3), (66, 511, 3), (66, 641, 3)])
def test_few_bytes(rows, k, out, layout, dtype):
    """Matrices shorter than what is read at a time, sums that end anywhere in it, and every number of stages up to six."""
    check((None, rows, k, out), dtype, "none", False, False, False, layout, seed=k)
    check(([rows - 1, 0, 1], 0, k, out), dtype, "none", False, False, False, layout, seed=k)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,k", [(3, 256), (40, 300), (300, 384)])
def test_codes_that_are_no_number_stay_in_their_row_and_column(dtype, rows, k):
    g = gen(k)
    xq, xs = codes(g, rows, k)
    wq, _ = codes(g, 70, k)
    ws = torch.full((1, xs.shape[1]), 127, device=DEV)
    xq[1, 5] = math.nan
    wq[17, k - 1] = math.nan
    y = moe.linear8(xq, bref.wide(xs), wq, bref.wide(ws), dtype=dtype)
    bad = torch.zeros(rows, 70, dtype=torch.bool, device=DEV)
    bad[1], bad[:, 17] = True, True
    assert torch.equal(torch.isnan(y), bad)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [5, 40, 300])
def test_scales_far_apart(dtype, rows):
    """Powers of two from 2^-60 to 2^60 meet their inverses."""
    g = gen(rows)
    k = 1280
    xq, xs = codes(g, rows, k)
    wq, _ = codes(g, 130, k)
    ws = torch.randint(67, 187, (2, 10), generator=g, device=DEV)
    xs = 254 - ws[0][None].expand(rows, 10) + torch.randint(-3, 3, (rows, 10), generator=g, device=DEV)
    ws = torch.stack([ws[0], ws[0]])
    y = moe.linear8(xq, bref.wide(xs), wq, bref.wide(ws), dtype=dtype)
    want, err = bref.product8(xq.double(), xs, wq.double(), ws, dtype)
    ref.close(y, want, err, dtype)


def test_a_long_sum_keeps_its_bits():
    """Binary32 results of 65536 products."""
    g = gen(9)
    xq, xs = codes(g, 40, 65536)
    wq, _ = codes(g, 64, 65536)
    ws = torch.full((1, 512), 120, device=DEV)
    y = moe.linear8(xq, bref.wide(xs), wq, bref.wide(ws), dtype=F32)
    want, err = bref.product8(xq.double(), xs, wq.double(), ws, F32)
    ref.close(y, want, err, F32)


def test_the_way_of_a_layer():
    """Rows and weights through quantise, the product, and its gradient on the
    transposed weight, against the same in 64 bits from the codes."""
    g = gen(4)
    counts = [40, 0, 17, 71]
    n, i, o = sum(counts), 264, 392
    off = torch.tensor([0, 40, 40, 57, 128], dtype=torch.int32, device=DEV)
    x, w = randn(g, n, i, dtype=BF16), randn(g, 4, o, i) * i ** -0.5
    xq, xs = moe.quantise(x, offsets=off)
    wq, ws = moe.quantise_weight(w)
    y = moe.linear8(xq, xs, wq, ws, offsets=off, act="silu")
    dy = randn(g, n, o, dtype=BF16)
    dq, ds = moe.quantise(dy, offsets=off)
    wt, wts = moe.quantise_weight(w, transpose=True)
    dx = moe.linear8(dq, ds, wt, wts, offsets=off)
    u8 = lambda t: t.view(torch.uint8)  # noqa: E731
    assert torch.equal(u8(wt), u8(wq).transpose(1, 2)) and torch.equal(u8(wts), u8(ws).transpose(1, 2))
    for gi, lo, hi in ref.spans(off, n):
        zz, ez = bref.product8(xq[lo:hi].double(), u8(xs)[lo:hi].long(), wq[gi].double(), u8(ws)[gi].long(), BF16)
        ref.close(y[lo:hi], ref.act(zz, "silu"), ref.act_err(zz, ez, "silu"), BF16)
        dd, ed = bref.product8(dq[lo:hi].double(), u8(ds)[lo:hi].long(), wt[gi].double(), u8(wts)[gi].long(), BF16)
        ref.close(dx[lo:hi], dd, ed, BF16)
        # and the unquantised product is near: codes are off by 2^-4 at most
        full = x[lo:hi].double() @ w[gi].double().t()
        assert hi == lo or float((zz - full).norm() / full.norm()) < 2 * 2.0 ** -4


def test_residual_in_place_a_stream_and_a_graph():
    g = gen(8)
    xq, xs = codes(g, 100, 384)
    wq, _ = codes(g, 256, 384)
    ws = bref.wide(torch.full((2, 3), 120, device=DEV))
    xs = bref.wide(xs)
    res = randn(g, 100, 256, dtype=BF16)
    want = moe.linear8(xq, xs, wq, ws, residual=res)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = res.clone()
    torch.cuda.synchronize()
    moe.linear8(xq, xs, wq, ws, residual=y, out=y, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    held, out = torch.zeros_like(xq), torch.zeros_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moe.linear8(held, xs, wq, ws, residual=res, out=out)
    for seed in range(4):
        held.copy_(codes(gen(seed), 100, 384)[0])
        graph.replay()
        again = moe.linear8(held, xs, wq, ws, residual=res)
        torch.cuda.synchronize()
        assert torch.equal(out, again)


def test_split_sums_do_not_depend_on_the_run():
    g = gen(6)
    xq, xs = codes(g, 48, 7168)
    wq, _ = codes(g, 130, 7168)
    xs, ws = bref.wide(xs), bref.wide(torch.full((2, 56), 121, device=DEV))
    first = moe.linear8(xq, xs, wq, ws, dtype=F32)
    for _ in range(5):
        torch.empty(1 << 22, dtype=torch.uint8, device=DEV).fill_(0xFF)
        assert torch.equal(moe.linear8(xq, xs, wq, ws, dtype=F32), first)


def test_refusals():
    g = gen(1)
    xq, xs = codes(g, 4, 200)
    wq, _ = codes(g, 64, 200)
    xs, ws = bref.wide(xs), bref.wide(torch.full((1, 2), 127, device=DEV))
    ok = moe.linear8(xq, xs, wq, ws)
    assert ok.dtype is BF16
    bad = [dict(x=xq.float()), dict(w=wq.float()), dict(x_scales=xs.float()), dict(x_scales=xs[:, :1]),
           dict(w_scales=bref.wide(torch.full((2, 2), 127, device=DEV))), dict(x=xq[:, :199]),
           dict(bias=torch.zeros(64, device=DEV)), dict(out=torch.zeros(4, 63, dtype=BF16, device=DEV)),
           dict(x_scales=torch.zeros(4, 2, dtype=torch.uint8, device=DEV).view(moe.E8M0)),
           dict(x_scales=torch.zeros(4, 2, dtype=torch.uint8).view(moe.E8M0)),
           dict(residual=torch.zeros(4, 64, dtype=BF16, device=DEV).requires_grad_()),
           # one row whose four scales are not all there
           dict(x=xq[:1], x_scales=torch.full((1, 2), 127, dtype=torch.uint8, device=DEV).view(moe.E8M0))]
    for kw in bad:
        args = dict(x=xq, x_scales=xs, w=wq, w_scales=ws)
        args.update(kw)
        with pytest.raises(ValueError):
            moe.linear8(**args)
    with pytest.raises(ll.LLError):
        moe.linear8(xq, xs, wq, ws, dtype=torch.float16)
    assert moe.linear8(xq[:0], xs[:0], wq, ws).shape == (0, 64)
