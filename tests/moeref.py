"""Plain 64-bit forms of the expert-layer operators, and the error bounds the
GPU tests hold the kernels to.

EPS is the unit in the last place of 1 in binary32 (2^-23, twice the rounding
error): a sum of n terms is off by at most n * EPS * sum |terms| whatever the
order, and a stored value by half a unit of its type, HALF[dtype] relative.
"""
import math

import torch

EPS = 2.0 ** -23
HALF = {dt: torch.finfo(dt).eps / 2 for dt in (torch.float32, torch.bfloat16)}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126}
GATED = ("swiglu", "geglu")


def one(z, act):
    """(f(z), f'(z)) of an ungated activation, float64."""
    if act in ("gelu", "geglu"):
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act in ("silu", "swiglu"):
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    return z, torch.ones_like(z)


def act(z, name):
    if name in GATED:
        a, u = z.chunk(2, -1)
        return one(a, name)[0] * u
    return one(z, name)[0]


def act_err(z, ez, name):
    """Bound on the error of act(z) when z is off by at most ez: the slopes of
    the activations stay within 1.13 and their binary32 evaluation is good to
    16 EPS of |z| (exp and erf are good to a few units, applied to values no
    larger than |z|)."""
    if name in GATED:
        a, u = z.chunk(2, -1)
        ea, eu = ez.chunk(2, -1)
        fa = 1.13 * ea + 16 * EPS * a.abs()
        return fa * (u.abs() + eu) + (one(a, name)[0].abs() + fa) * eu + EPS * (one(a, name)[0] * u).abs()
    return 1.13 * ez + (16 * EPS * z.abs() if name != "none" else 0)


def through(g, z, name):
    """The gradient g of act(z), taken to z."""
    if name == "none":
        return g
    if name in GATED:
        a, u = z.chunk(2, -1)
        f, s = one(a, name)
        return torch.cat([g * u * s, g * f], -1)
    return g * one(z, name)[1]


def through_err(g, eg, z, name):
    """Bound on the error of through(g, z) when g is off by eg: slopes within
    1.13, evaluated to 32 EPS (1 + |z|); values within |z|, to 16 EPS |z|."""
    if name == "none":
        return eg
    if name in GATED:
        a, u = z.chunk(2, -1)
        es = 32 * EPS * (1 + a.abs())
        ef = 16 * EPS * a.abs()
        return torch.cat([(1.13 * eg + g.abs() * es) * u.abs() + 4 * EPS * (g * u).abs(),
                          eg * (a.abs() + ef) + g.abs() * ef + 4 * EPS * (g * a).abs()], -1)
    return 1.13 * eg + g.abs() * 32 * EPS * (1 + z.abs())


def close(got, want, err, dtype):
    """got (dtype) against want (float64), computed to within err before it was rounded."""
    bound = err + (want.abs() + err) * HALF[dtype] * 1.01 + TINY[dtype]
    bad = ~((got.double() - want).abs() <= bound)
    if bool(bad.any()):
        at = bad.nonzero()[0].tolist()
        i = tuple(at)
        raise AssertionError(f"{int(bad.sum())} of {bad.numel()} values off, first at {at}: got {got[i].item()}, "
                             f"expected {want[i].item()} within {bound[i].item()}")


def spans(offsets, rows):
    if offsets is None:
        return [(0, 0, rows)]
    b = offsets.tolist()
    return [(g, b[g], b[g + 1]) for g in range(len(b) - 1)]


def matmul(a, b):
    """(a b, a bound on its binary32 error), float64."""
    n = a.shape[1]
    return a @ b, (n + 4) * EPS * (a.abs() @ b.abs())


def sort(ids, first, experts):
    """(offsets, slots, rows) of a stable sort by local expert, by counting in Python."""
    t, k = ids.shape
    flat = ids.reshape(-1).tolist()
    order = [i for e in range(first, first + experts) for i, v in enumerate(flat) if v == e]
    offsets = [0]
    for e in range(first, first + experts):
        offsets.append(offsets[-1] + flat.count(e))
    rows = [-1] * len(flat)
    for place, i in enumerate(order):
        rows[i] = place
    return offsets, order + [-1] * (len(flat) - len(order)), torch.tensor(rows, dtype=torch.int32).reshape(t, k)


def route(logits, bias, k, score, normalise, scale):
    """(ids, weights, scores, total) for float64 logits whose keys are binary32 sums."""
    key = logits.float() if bias is None else logits.float() + bias
    key = torch.where(torch.isnan(key), torch.full_like(key, -math.inf), key).cpu()
    ids = torch.full((logits.shape[0], k), -1, dtype=torch.int64)
    for t, row in enumerate(key.tolist()):
        order = sorted((i for i, v in enumerate(row) if v > -math.inf), key=lambda i: (-row[i], i))[:k]
        ids[t, :len(order)] = torch.tensor(order, dtype=torch.int64)
    ids = ids.to(logits.device)
    l = torch.where(torch.isnan(logits), torch.full_like(logits, -math.inf), logits)
    if score == "softmax":
        p = torch.softmax(l, 1)
        p = torch.where(torch.isnan(p), torch.zeros_like(p), p)
    else:
        p = torch.sigmoid(l)
    u = torch.where(ids >= 0, p.gather(1, ids.clamp(min=0)), torch.zeros_like(p[:, :1]))
    if normalise:
        tot = u.sum(1, keepdim=True)
        u = torch.where(tot > 0, u / torch.where(tot > 0, tot, torch.ones_like(tot)), torch.zeros_like(u))
    return ids, scale * u
