"""Plain forms of the 8-bit values, the 8-bit products, the norms and the
weight update, and the error bounds the GPU tests hold the kernels to.

Codes and scales are exact: a scale is a power of two, a value times its
inverse is exact in 64 bits, and the rounding is to nearest, ties to even.
"""
import numpy as np
import torch

import moeref as ref

EPS = ref.EPS
E4M3, E5M2, E8M0 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
BLOCK = 128


def two(e):
    """2^e in 64 bits, from its bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def exponents(amax, top=8):
    """Scale codes (exponent + 127): the least power of two with amax <= 1.75 * 2^top of it, at least 2^-126."""
    frac, e = torch.frexp(amax.double())  # frac in [1/2, 1)
    s = e - (top + 1) + (frac > 0.875).to(e.dtype)
    return torch.where(amax > 0, s + 127, torch.ones_like(s)).clamp(min=1)


def round_e4m3(y):
    """The nearest e4m3 value, ties to even; what is not finite becomes NaN."""
    step = two(torch.frexp(y)[1].clamp(min=-5) - 4)
    return torch.where(torch.isfinite(y), torch.round(y / step) * step, torch.full_like(y, float("nan")))


def finite(x):
    return torch.where(torch.isfinite(x), x, torch.zeros_like(x)).abs()


def quantise(x):
    """(values [n, h], scale codes [n, blocks]) of float64 rows."""
    parts = x.split(BLOCK, 1)
    codes = torch.stack([exponents(finite(p).amax(1)) for p in parts], 1)
    q = torch.cat([round_e4m3(p / two(codes[:, i:i + 1] - 127)) for i, p in enumerate(parts)], 1)
    return q, codes


def quantise_weight(w):
    """(values [out, in], scale codes) of one float64 weight."""
    q, codes = torch.empty_like(w), []
    for i, strip in enumerate(w.split(BLOCK, 0)):
        row = []
        for j, p in enumerate(strip.split(BLOCK, 1)):
            c = exponents(finite(p).amax())
            row.append(c)
            q[i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK] = round_e4m3(p / two(c - 127))
        codes.append(torch.stack(row))
    return q, torch.stack(codes)


def wide(scales):
    """Scale codes (whole numbers) in memory whose rows start at multiples of 4."""
    pad = (scales.shape[-1] + 3) // 4 * 4
    buf = torch.full((*scales.shape[:-1], pad), 255, dtype=torch.uint8, device=scales.device)  # no number in the padding
    buf[..., :scales.shape[-1]] = scales.to(torch.uint8)
    return buf.view(E8M0)[..., :scales.shape[-1]]


def same_values(got, want):
    """Codes `got` stand for exactly `want` (NaN for NaN)."""
    g = got.double()
    assert torch.equal(torch.isnan(g), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(g, nan=0.0), torch.nan_to_num(want, nan=0.0))


def stretch(codes, n, dim):
    """A scale (from codes) for each value along dim."""
    return two(codes.to(torch.int64) - 127).repeat_interleave(BLOCK, dim).narrow(dim, 0, n)


def tops(q, codes, dim_scale):
    """For each row and eight consecutive k: the largest magnitude, no less than that of the least normal code."""
    n, k = q.shape
    s = dim_scale
    mag = torch.maximum(q.abs(), torch.full_like(q, 2.0 ** -6)) * s
    pad = (-k) % 8
    return torch.nn.functional.pad(mag, (0, pad)).view(n, (k + pad) // 8, 8).amax(2)


def product8(xq, xc, wq, wc, dtype):
    """(x w^T, a bound on its error) in float64, for values and scale codes.

    Binary32 results: sums of k terms, (k + 4) EPS of the sum of magnitudes.
    bfloat16 results besides: of eight consecutive products all but the largest
    may lose 2^-13 of the largest one's power of two."""
    k = xq.shape[1]
    sx, sw = stretch(xc, k, 1), stretch(stretch_rows(wc, wq.shape[0]), k, 1)
    x, w = xq * sx, wq * sw
    err = (k + 4) * EPS * (x.abs() @ w.abs().t())
    if dtype is torch.bfloat16:
        err = err + 7 * 2.0 ** -13 * (tops(xq, xc, sx) @ tops(wq, wc, sw).t())
    return x @ w.t(), err


def stretch_rows(codes, n):
    return codes.repeat_interleave(BLOCK, 0)[:n]


# ---------------------------------------------------------------- norms
def rstd(x, eps):
    return 1 / torch.sqrt(x.square().mean(1, keepdim=True) + eps)


def norm(y, x, gate, scale, post, weight, eps):
    """(h, r) in float64 and a bound on the binary32 error of each.

    A sum of n squares is relatively off by n EPS at most, so is its root by
    half of that; every further operation adds EPS."""
    n = y.shape[1]
    rel = (n / 2 + 8) * EPS
    u, eu = y, torch.zeros_like(y)
    if post is not None:
        u = y * rstd(y, eps) * post
        eu = rel * u.abs()
    by = scale * (gate[:, None] if gate is not None else 1.0)
    r = by * u
    er = (eu * abs(scale) * (gate[:, None].abs() if gate is not None else 1.0)) + 3 * EPS * r.abs()
    if x is not None:
        r = r + x
        er = er + EPS * r.abs()
    if weight is None:
        return None, None, r, er
    rs = rstd(r, eps)
    h = r * rs * weight
    # the root's argument moves with r's error
    drift = rs * torch.sqrt(er.square().mean(1, keepdim=True))
    return h, (weight * rs).abs() * er + h.abs() * (rel + drift), r, er


def norm_back(d, ed, x, w, eps):
    """x -> x rstd(x) w backwards: (dx, its error, dw, its error) for a gradient d off by ed."""
    n, rows = x.shape[1], x.shape[0]
    rel = (n + 16) * EPS
    rs = rstd(x, eps)
    u = x * rs
    g, eg = w * d, w.abs() * ed
    m = (g * u).mean(1, keepdim=True)
    em = (eg * u.abs()).mean(1, keepdim=True) + 2 * rel * (g * u).abs().mean(1, keepdim=True)
    dx = rs * (g - u * m)
    ex = rs * (eg + u.abs() * em) + 2 * rel * rs * (g.abs() + (u * m).abs())
    return dx, ex, (d * u).sum(0), (ed * u.abs()).sum(0) + (2 * rel + rows * EPS) * (d * u).abs().sum(0)


def norm_grad(dh, r, dr, y, gate, scale, post, weight, eps):
    """{name: (value, bound)} of norm's gradients, float64."""
    out = {}
    d = torch.zeros_like(r if r is not None else dr)
    ed = torch.zeros_like(d)
    if weight is not None:
        d, ed, dw, ew = norm_back(dh, torch.zeros_like(dh), r, weight, eps)
        out["dweight"] = (dw, ew)
    if dr is not None:
        d = d + dr
        ed = ed + EPS * d.abs()
    out["dr"] = (d, ed)
    n = d.shape[1]
    u = y
    if post is not None:
        u = y * rstd(y, eps) * post
    if gate is not None:
        out["dgate"] = (scale * (d * u).sum(1),
                        abs(scale) * ((ed * u.abs()).sum(1) + 2 * (n + 16) * EPS * (d * u).abs().sum(1)))
    by = scale * (gate[:, None] if gate is not None else torch.ones_like(d[:, :1]))
    g, eg = by * d, by.abs() * ed + 2 * EPS * (by * d).abs()
    if post is not None:
        g, eg, dp, ep = norm_back(g, eg, y, post, eps)
        out["dpost"] = (dp, ep)
    out["dy"] = (g, eg)
    return out


# ---------------------------------------------------------------- the weight update
def mix(x):
    x = np.asarray(x, dtype=np.uint64) & 0xFFFFFFFF
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x7FEB352D)) & np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x846CA68B)) & np.uint64(0xFFFFFFFF)
    return x ^ (x >> np.uint64(16))


def random_bits(first, n, step, seed):
    """The 32-bit number of each of n values from number `first` on."""
    at = np.arange(first, first + n, dtype=np.uint64)
    key = mix((seed + step * 0x9E3779B9) & 0xFFFFFFFF)
    high = ((at >> np.uint64(32)) * np.uint64(0x9E3779B9)) & np.uint64(0xFFFFFFFF)
    return mix((at & np.uint64(0xFFFFFFFF)) ^ high ^ key)


def block_scales(x, top):
    """Scale codes of float32 values in blocks of 128, from their bits."""
    n = len(x)
    pad = np.zeros((n + BLOCK - 1) // BLOCK * BLOCK, dtype=np.float32)
    pad[:n] = np.where(np.isfinite(x), np.abs(x), 0)
    bits = pad.reshape(-1, BLOCK).max(1).view(np.uint32).astype(np.int64)
    return np.maximum((bits >> 23) - top + ((bits & 0x7FFFFF) > 0x600000), 1)


def stochastic(x, codes, r, mant, emin, bias):
    """8-bit codes of float32 x, rounded up where the random bits carry."""
    inv = ((254 - np.repeat(codes, BLOCK)[:len(x)]) << 23).astype(np.uint32).view(np.float32)
    y = x * inv
    cut = 23 - mant
    bits = np.abs(y).view(np.uint32).astype(np.int64)
    r = r.astype(np.int64)
    fine = ((bits + r) >> cut) - ((127 - bias) << mant)
    mag = np.abs(y).astype(np.float64)
    low = (np.minimum(mag * 2.0 ** (mant - emin + cut), 2.0 ** 23).astype(np.int64) + r) >> cut
    code = np.where(mag < 2.0 ** emin, low, fine)
    code = np.where(np.isfinite(y), code | (np.signbit(y).astype(np.int64) << 7), 0x7F)
    return code.astype(np.uint8)


def adamw_states(m, v, g, beta1, beta2):
    """The new m and v, operation by operation in binary32."""
    f = np.float32
    m = m * f(beta1) + g * f(1 - beta1)
    v = v * f(beta2) + (g * g) * f(1 - beta2)
    return m, v
