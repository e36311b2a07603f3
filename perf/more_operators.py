"""Performance cases of the 8-bit expert products, the norms around a block and
the weight update.

A case names an operation ("op") and its sizes:

  quantise         "rows" x "features" to e4m3 with a power-of-two scale for each
                   128 features of a row, through "act" first (gated ones halve
                   the features that come in); "tail": the buffer has that many
                   rows behind the last group's
  quantise_weight  "groups" weights [out, in] in blocks of 128 x 128;
                   "transpose": the codes come out as [in, out]
  linear8          rows in "groups" groups times each group's weight, both in 8
                   bits; "act", and where they say so a bias, a residual row and
                   the pre-activations; "dtype" is the output's
  norm             "tokens" x "features": a block's output through its own norm
                   ("post"), times the token's "gate", added to the residual
                   stream, and the next block's norm of that; "q": the normed
                   rows in 8 bits too
  norm_grad        the gradients of all of that
  adamw            a step over "layers" x 5 tensors (two norm weights, a router,
                   the experts' up- and down-projections) with "bits" a state
                   value; "grad": the gradients' type

``own`` selects the framework's kernels; otherwise the plain forms run.
"""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
GATED = ("swiglu", "geglu")
E4M3, E5M2, E8M0 = torch.float8_e4m3fn, torch.float8_e5m2, torch.float8_e8m0fnu
BLOCK = 128
EPS = 1e-6                                                         # of the norms
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.95, 1e-8, 0.1      # of the update
SEED = 1234567                                                     # of its random rounding


# ---------------------------------------------------------------- cases
def listed():
    return [
        # decode, batch 16 at hidden 7168: the rows of one product
        {"name": "quantise_b16", "op": "quantise", "rows": 16, "features": 7168, "dtype": "bf16", "act": "none", "tail": 0},
        # prefill: the experts' gated pre-activations on their way into the down-projection, in a buffer with room
        {"name": "quantise_swiglu_prefill", "op": "quantise", "rows": 16384, "features": 2048, "dtype": "bf16",
         "act": "swiglu", "tail": 4096},
        # training: 8 experts' down-projections, from their binary32 masters, for the gradient of the rows
        {"name": "quantise_weight_transposed", "op": "quantise_weight", "groups": 8, "out": 7168, "in": 2048,
         "dtype": "f32", "transpose": True},
        # decode, batch 16: about one row for every second expert; the weights stream
        {"name": "linear8_decode", "op": "linear8", "rows": 16, "groups": 32, "in": 7168, "out": 4096, "dtype": "bf16",
         "act": "swiglu", "bias": False, "residual": False, "save": False},
        # training: the gradient of the down-projections' rows, on their transposed weights
        {"name": "linear8_grad_x", "op": "linear8", "rows": 8192, "groups": 8, "in": 7168, "out": 2048, "dtype": "bf16",
         "act": "none", "bias": False, "residual": False, "save": False},
        # prefill: 16384 rows over 32 experts, the gated up-projection (the largest)
        {"name": "linear8_prefill", "op": "linear8", "rows": 16384, "groups": 32, "in": 7168, "out": 4096,
         "dtype": "bf16", "act": "swiglu", "bias": False, "residual": False, "save": False},
        # odd sizes, binary32 out, pre-activations kept for the way back
        {"name": "linear8_odd", "op": "linear8", "rows": 777, "groups": 5, "in": 1001, "out": 515, "dtype": "f32",
         "act": "gelu", "bias": True, "residual": True, "save": True},
        # decode, batch 16: everything between two blocks, with the next product's rows
        {"name": "norm_b16", "op": "norm", "tokens": 16, "features": 7168, "dtype": "bf16", "post": True, "gate": True,
         "residual": True, "q": True},
        # training: a residual stream of 8192 tokens
        {"name": "norm_train", "op": "norm", "tokens": 8192, "features": 7168, "dtype": "bf16", "post": False,
         "gate": False, "residual": True, "q": False},
        # and its way back with a norm and a gate on the block's output
        {"name": "norm_grad_train", "op": "norm_grad", "tokens": 8192, "features": 7168, "dtype": "bf16", "post": True,
         "gate": True, "residual": True},
        # many tensors of odd sizes, states in binary32
        {"name": "adamw_many", "op": "adamw", "layers": 8, "hidden": 501, "ffn": 203, "experts": 4, "dtype": "f32",
         "grad": "f32", "bits": 32},
        # a rank's experts: 8 of hidden 7168, states in 8 bits
        {"name": "adamw_experts_8bit", "op": "adamw", "layers": 1, "hidden": 7168, "ffn": 2048, "experts": 8,
         "dtype": "bf16", "grad": "f32", "bits": 8},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A feature count: mostly multiples of 8, as models have, some odd."""
    n = _log(rng, lo, hi)
    return n if rng.random() < 0.25 else max(8, n // 8 * 8)


def draw(rng):
    op = rng.choice(["quantise", "quantise_weight", "linear8", "linear8", "norm", "norm_grad", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    acts = ["none", "none", "relu", "gelu", "silu", "swiglu", "geglu"]
    case = {"op": op, "dtype": dtype}
    if op == "quantise":
        case.update(rows=_log(rng, 1, 16384), features=_size(rng, 64, 8192), act=rng.choice(acts))
        case["tail"] = rng.choice([0, 0, 1 + case["rows"] // 3])
    elif op == "quantise_weight":
        case.update(groups=rng.choice([1, 1, 4, 8, 32]), out=_size(rng, 64, 7168), transpose=rng.random() < 0.5)
        case["in"] = _size(rng, 64, 7168)
        while case["groups"] * case["out"] * case["in"] > 120e6:  # no dearer than the listed one
            case["groups"] = (case["groups"] + 1) // 2
    elif op == "linear8":
        case.update(rows=_log(rng, 1, 16384), groups=rng.choice([1, 1, 4, 8, 16, 32]), out=_size(rng, 64, 7168) // 2 * 2)
        case["in"] = _size(rng, 64, 7168)
        case["act"] = rng.choice(acts)
        case.update(bias=rng.random() < 0.5, residual=rng.random() < 0.5, save=rng.random() < 0.3)
        while _flops(case) > 9e11:  # no dearer than the largest listed one
            case["rows"] = max(1, case["rows"] // 2)
    elif op in ("norm", "norm_grad"):
        case.update(tokens=_log(rng, 1, 8192), features=_size(rng, 64, 7168), post=rng.random() < 0.5,
                    gate=rng.random() < 0.5, residual=rng.random() < 0.8)
        if dtype == "f32":
            case["tokens"] = min(case["tokens"], 4096)
        if op == "norm":
            case["q"] = rng.random() < 0.4
    else:
        case.update(layers=rng.randint(1, 8), hidden=_size(rng, 64, 7168), ffn=_size(rng, 64, 2048),
                    experts=rng.choice([1, 2, 4, 8]), grad=rng.choice(["f32", "f32", "bf16"]), bits=rng.choice([8, 32]))
        while _parameters(case) > (352e6 if case["bits"] == 8 and dtype == "bf16" else 230e6):
            if case["layers"] > 1:
                case["layers"] //= 2
            else:
                case["experts"] = max(1, case["experts"] // 2)
    return case


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _hidden(g, n, h):
    """Hidden rows: some features and some rows are much larger than others."""
    return _randn(g, n, h) * torch.exp(0.7 * _randn(g, 1, h)) * torch.exp(0.3 * _randn(g, n, 1))


def _offsets(g, rows, groups):
    """[groups + 1] offsets of `rows` rows that chose among the groups with
    uneven liking; few rows leave groups empty."""
    p = torch.softmax(0.5 * _randn(g, groups), 0)
    pick = torch.multinomial(p, rows, replacement=True, generator=g)
    off = torch.zeros(groups + 1, dtype=torch.int32, device="cuda")
    off[1:] = torch.cumsum(torch.bincount(pick, minlength=groups), 0)
    return off


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _scales(*shape):
    """Memory for scales: a row of them starts at a multiple of 4."""
    wide = torch.zeros(*shape[:-1], (shape[-1] + 3) // 4 * 4, dtype=torch.uint8, device="cuda")
    return wide.view(E8M0)[..., :shape[-1]]


def _put_scales(values):
    s = _scales(*values.shape)
    s.view(torch.uint8).copy_(values.view(torch.uint8))
    return s


def _shapes(case):
    """(shape, type) of each tensor that an update goes over."""
    e, h, f, dt = case["experts"], case["hidden"], case["ffn"], TORCH[case["dtype"]]
    one = [((h,), torch.float32), ((h,), torch.float32), ((8 * e, h), torch.float32), ((e, 2 * f, h), dt), ((e, h, f), dt)]
    return one * case["layers"]


def _parameters(case):
    e, h, f = case["experts"], case["hidden"], case["ffn"]
    return case["layers"] * (2 * h + 8 * e * h + 3 * e * f * h)


def _padded(n):
    return _blocks(n) * BLOCK


def _adamw_inputs(case, g):
    shapes = _shapes(case)
    sizes = [math.prod(shape) for shape, _ in shapes]
    total = sum(_padded(n) for n in sizes)
    size = torch.exp(torch.linspace(-9, -3, len(shapes), device="cuda"))  # of the tensors' gradients
    place = torch.cat([z.expand(_padded(n)) for z, n in zip(size, sizes)])
    here = torch.cat([torch.arange(_padded(n), device="cuda") < n for n in sizes])
    masters = [0.05 * _randn(g, *shape) for shape, _ in shapes]
    s = {"params": [w.to(dt) for w, (_, dt) in zip(masters, shapes)],
         "masters": [w if dt == torch.bfloat16 else None for w, (_, dt) in zip(masters, shapes)],
         "grads": [(scale * _randn(g, *shape)).to(TORCH[case["grad"]]) for scale, (shape, _) in zip(size, shapes)],
         "sizes": sizes, "count": torch.full((1,), 40, dtype=torch.int32, device="cuda")}
    m = torch.where(here, 0.3 * place * _randn(g, total), 0.0)
    v = torch.where(here, (place * (0.2 + _randn(g, total).abs())) ** 2, 0.0)
    if case["bits"] == 8:
        s["m"], s["m_scales"] = _flat8(m, E4M3, 8)
        s["v"], s["v_scales"] = _flat8(v, E5M2, 15)
    else:
        s["m"], s["v"], s["m_scales"], s["v_scales"] = m, v, None, None
    return s


def _flat8(x, dtype, top):
    b = x.view(-1, BLOCK)
    code = _exponent(b.abs().amax(1), top)
    return (b * _power(127 - code)[:, None]).to(dtype).view(-1), code.to(torch.uint8).view(E8M0)


def _inputs(case, seed):
    g = _gen(seed)
    op, dt = case["op"], TORCH[case["dtype"]]
    s = {"case": case}
    if op == "quantise":
        n, h = case["rows"] + case["tail"], case["features"]
        s["x"] = _hidden(g, n, h * (2 if case["act"] in GATED else 1)).to(dt)
        s["offsets"] = torch.tensor([0, case["rows"]], dtype=torch.int32, device="cuda") if case["tail"] else None
        s["q"] = torch.zeros(n, h, dtype=torch.uint8, device="cuda").view(E4M3)
        s["scales"] = _scales(n, _blocks(h))
    elif op == "quantise_weight":
        groups, o, i = case["groups"], case["out"], case["in"]
        s["w"] = (_randn(g, groups, o, i) * i ** -0.5).to(dt)
        if case["transpose"]:
            o, i = i, o
        s["q"] = torch.zeros(groups, o, i, dtype=torch.uint8, device="cuda").view(E4M3)
        s["scales"] = _scales(groups, _blocks(o), _blocks(i))
    elif op == "linear8":
        n, groups, ki, mo = case["rows"], case["groups"], case["in"], case["out"]
        width = _out_width(case)
        s["offsets"] = _offsets(g, n, groups)
        s["bounds"] = s["offsets"].tolist()
        s["x"], scales = _quantise(_hidden(g, n, ki))
        s["x_scales"] = _put_scales(scales)
        w = [_quantise_blocks(_randn(g, 1, mo, ki) * ki ** -0.5) for _ in range(groups)]
        s["w"], s["w_scales"] = torch.cat([q for q, _ in w]), _put_scales(torch.cat([c.view(torch.uint8) for _, c in w]))
        s["b"] = (0.2 * _randn(g, groups, mo)).to(dt) if case["bias"] else None
        s["residual"] = _randn(g, n, width).to(dt) if case["residual"] else None
        s["out"] = torch.zeros(n, width, dtype=dt, device="cuda")
        s["z"] = torch.zeros(n, mo, dtype=dt, device="cuda") if case["save"] else None
    elif op in ("norm", "norm_grad"):
        n, h = case["tokens"], case["features"]
        s["weight"] = (1 + 0.2 * _randn(g, h)).to(dt)
        s["post"] = (1 + 0.2 * _randn(g, h)).to(dt) if case["post"] else None
        s["gate"] = torch.sigmoid(_randn(g, n)) if case["gate"] else None
        s["scale"] = 0.5 if case["residual"] else 1.0
        s["y"] = _hidden(g, n, h).to(dt)
        if op == "norm":
            s["residual"] = (3 * _hidden(g, n, h)).to(dt) if case["residual"] else None
            s["h"], s["r"] = torch.zeros_like(s["y"]), torch.zeros_like(s["y"])
            if case["q"]:
                s["q"] = torch.zeros(n, h, dtype=torch.uint8, device="cuda").view(E4M3)
                s["scales"] = _scales(n, _blocks(h))
        else:
            s["r"] = (3 * _hidden(g, n, h)).to(dt)
            s["dh"] = _randn(g, n, h).to(dt)
            s["dr"] = _randn(g, n, h).to(dt)
            s["dr_out"], s["dy"] = torch.zeros_like(s["y"]), torch.zeros_like(s["y"])
            s["dgate"] = torch.zeros_like(s["gate"]) if case["gate"] else None
            s["dweight"] = torch.zeros(h, dtype=torch.float32, device="cuda")
            s["dpost"] = torch.zeros(h, dtype=torch.float32, device="cuda") if case["post"] else None
    else:
        s.update(_adamw_inputs(case, g))
    return s


def _out_width(case):
    return case["out"] // 2 if case["act"] in GATED else case["out"]


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and case["op"] == "adamw":  # the handle that a training program keeps, on the state that is there
        from paper_2607_16100_amd.optim import AdamW

        s["opt"] = AdamW(s["params"], lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=DECAY,
                         states="8bit" if case["bits"] == 8 else "f32", seed=SEED,
                         state={k: s[k] for k in ("masters", "m", "v", "m_scales", "v_scales", "count")})
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2607_16100_amd import moe

    case = s["case"]
    op = case["op"]
    if op == "quantise":
        return moe.quantise(s["x"], act=case["act"], offsets=s["offsets"], out=s["q"], scales=s["scales"])
    if op == "quantise_weight":
        return moe.quantise_weight(s["w"], transpose=case["transpose"], out=s["q"], scales=s["scales"])
    if op == "linear8":
        y = moe.linear8(s["x"], s["x_scales"], s["w"], s["w_scales"], bias=s["b"], act=case["act"],
                        residual=s["residual"], offsets=s["offsets"], out=s["out"], z=s["z"])
        return (y, s["z"]) if case["save"] else y
    if op == "norm":
        got = moe.norm(s["y"], s["weight"], residual=s["residual"], gate=s["gate"], scale=s["scale"], post=s["post"],
                       eps=EPS, h=s["h"], r=s["r"], q=s.get("q"), q_scales=s.get("scales"))
        return tuple(t for t in got if t is not None)
    if op == "norm_grad":
        got = moe.norm_grad(s["dh"], s["r"], s["weight"], dr=s["dr"], y=s["y"], gate=s["gate"], scale=s["scale"],
                            post=s["post"], eps=EPS, dr_out=s["dr_out"], dy=s["dy"], dgate=s["dgate"],
                            dweight=s["dweight"], dpost=s["dpost"])
        return tuple(t for t in got if t is not None)
    s["opt"].step(s["grads"])
    return _adamw_outputs(s)


def _adamw_outputs(s):
    return ([p.view(-1) for p in s["params"]], [w.view(-1) for w in s["masters"] if w is not None], s["m"], s["v"],
            s["m_scales"], s["v_scales"], s["count"])


# ---------------------------------------------------------------- plain forms
def _act(z, act):
    if act == "relu":
        return torch.clamp_min(z, 0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act in GATED:
        a, u = z.chunk(2, dim=-1)
        return _act(a, "silu" if act == "swiglu" else "gelu") * u
    return z


def _exponent(amax, top):
    """The exponent (biased by 127, in [1, 254]) of the least power of two with amax <= 1.75 * 2^top times it."""
    bits = amax.contiguous().view(torch.int32)
    return ((bits >> 23) - top + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(1, 254)


def _power(e):
    """2^e for whole e in [-126, 127]."""
    return ((e + 127) << 23).int().view(torch.float32)


def _quantise(x):
    """Rows of binary32 to (codes, scales), a scale for each 128 of a row."""
    n, h = x.shape
    b = torch.nn.functional.pad(x, (0, _padded(h) - h)).view(n, -1, BLOCK)
    code = _exponent(b.abs().amax(2), 8)
    q = (b * _power(127 - code)[:, :, None]).to(E4M3)
    return q.view(n, -1)[:, :h].contiguous(), code.to(torch.uint8).view(E8M0)


def _quantise_blocks(w):
    """Weights [groups, out, in] of binary32 to (codes, scales), a scale for each 128 x 128."""
    groups, o, i = w.shape
    b = torch.nn.functional.pad(w, (0, _padded(i) - i, 0, _padded(o) - o)).view(groups, -1, BLOCK, _blocks(i), BLOCK)
    code = _exponent(b.abs().amax((2, 4)), 8)
    q = (b * _power(127 - code)[:, :, None, :, None]).to(E4M3)
    return q.view(groups, _padded(o), -1)[:, :o, :i].contiguous(), code.to(torch.uint8).view(E8M0)


def _stretch(scales, n, dim):
    return scales.float().repeat_interleave(BLOCK, dim).narrow(dim, 0, n)


def _linear8(s, case):
    b, wq, ws = s["bounds"], s["w"], s["w_scales"]
    x = s["x"].float() * _stretch(s["x_scales"], case["in"], 1)

    def product(i):
        w = wq[i].float() * _stretch(_stretch(ws[i], case["out"], 0), case["in"], 1)
        return x[b[i]:b[i + 1]] @ w.t()

    z = torch.cat([product(i) for i in range(case["groups"]) if b[i] < b[i + 1]])
    if s["b"] is not None:
        counts = (s["offsets"][1:] - s["offsets"][:-1]).long()
        z = z + s["b"].float().repeat_interleave(counts, 0, output_size=case["rows"])
    y = _act(z, case["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    dt = TORCH[case["dtype"]]
    return (y.to(dt), z.to(dt)) if case["save"] else y.to(dt)


def _rstd(x):
    return torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)


def _norm(s, case):
    dt = TORCH[case["dtype"]]
    r = s["y"].float()
    if s["post"] is not None:
        r = r * _rstd(r) * s["post"].float()
    if s["gate"] is not None:
        r = r * s["gate"][:, None]
    r = r * s["scale"]
    if s["residual"] is not None:
        r = r + s["residual"].float()
    h = r * _rstd(r) * s["weight"].float()
    return (h.to(dt), r.to(dt)) + (_quantise(h) if case["q"] else ())


def _norm_back(dh, x, w):
    """(gradient of x, gradient of w) of x * rstd(x) * w."""
    rs = _rstd(x)
    n, g = x * rs, dh * w
    return rs * (g - n * (g * n).mean(1, keepdim=True)), (dh * n).sum(0)


def _norm_grad(s, case):
    dt = TORCH[case["dtype"]]
    dr, dweight = _norm_back(s["dh"].float(), s["r"].float(), s["weight"].float())
    dr = dr + s["dr"].float()
    y, post, gate = s["y"].float(), s["post"], s["gate"]
    u = y if post is None else y * _rstd(y) * post.float()
    dgate = None if gate is None else s["scale"] * (dr * u).sum(1)
    dy = s["scale"] * (dr if gate is None else dr * gate[:, None])
    dpost = None
    if post is not None:
        dy, dpost = _norm_back(dy, y, post.float())
    return tuple(t for t in (dr.to(dt), dy.to(dt), dgate, dweight, dpost) if t is not None)


def _mix(x):
    """A bijection of 32-bit numbers (held in 64 bits) whose every output bit depends on every input bit."""
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random(total, step):
    """A 32-bit number for each state value and step."""
    at = torch.arange(total, device="cuda")
    key = _mix((SEED + step.long() * 0x9E3779B9) & 0xFFFFFFFF)
    return _mix((at & 0xFFFFFFFF) ^ key)  # fewer than 2^32 values here


def _stochastic(y, r, mant, emin, dtype):
    """y to the format of `mant` mantissa bits and least normal exponent emin, up or down as the random r says."""
    cut = 23 - mant
    mag = y.abs()
    fine = ((mag.view(torch.int32) + r) >> cut << cut).int().view(torch.float32)
    sub = ((mag * 2.0 ** (mant - emin + cut)).clamp(max=2.0 ** 23).int() + r) >> cut
    low = sub.float() * 2.0 ** (emin - mant)
    return torch.copysign(torch.where(mag < 2.0 ** emin, low, fine), y).to(dtype)


def _to8(x, r, mant, emin, top, dtype):
    b = x.view(-1, BLOCK)
    code = _exponent(b.abs().amax(1), top)
    return (_stochastic((b * _power(127 - code)[:, None]).view(-1), r, mant, emin, dtype),
            code.to(torch.uint8).view(E8M0))


def _from8(q, scales):
    return (q.float().view(-1, BLOCK) * scales.float()[:, None]).view(-1)


def _adamw(s, case):
    eight = case["bits"] == 8
    flat = lambda ts: torch.cat([torch.nn.functional.pad(t.reshape(-1).float(), (0, _padded(n) - n))
                                 for t, n in zip(ts, s["sizes"])])
    s["count"] += 1
    t = s["count"].double()
    step, rden = (LR / (1 - BETA1 ** t)).float(), (1 / torch.sqrt(1 - BETA2 ** t)).float()
    g = flat(s["grads"])
    p = flat([q if w is None else w for q, w in zip(s["params"], s["masters"])])
    m, v = (_from8(s["m"], s["m_scales"]), _from8(s["v"], s["v_scales"])) if eight else (s["m"], s["v"])
    m = m * BETA1 + g * (1 - BETA1)
    v = v * BETA2 + g * g * (1 - BETA2)
    p = p * (1 - LR * DECAY) - step * m / (torch.sqrt(v) * rden + ADAM_EPS)
    if eight:
        r = _random(m.numel(), s["count"])
        new_m, new_ms = _to8(m, ((r >> 16) << 4).int(), 3, -6, 8, E4M3)
        new_v, new_vs = _to8(v, ((r & 0xFFFF) << 5).int(), 2, -14, 15, E5M2)
        s["m_scales"].view(torch.uint8).copy_(new_ms.view(torch.uint8))
        s["v_scales"].view(torch.uint8).copy_(new_vs.view(torch.uint8))
        s["m"].view(torch.uint8).copy_(new_m.view(torch.uint8))
        s["v"].view(torch.uint8).copy_(new_v.view(torch.uint8))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    parts = [w[:n].view(q.shape) for w, n, q in zip(p.split([_padded(n) for n in s["sizes"]]), s["sizes"], s["params"])]
    # one at a time: a copy of many at once takes the first tensor's type for all of them
    for q, w, x in zip(s["params"], s["masters"], parts):
        q.copy_(x)
        if w is not None:
            w.copy_(x)
    return _adamw_outputs(s)


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op == "quantise":
        n = case["rows"]
        q, scales = _quantise(_act(s["x"][:n].float(), case["act"]))
        s["q"].view(torch.uint8)[:n] = q.view(torch.uint8)
        s["scales"].view(torch.uint8)[:n] = scales.view(torch.uint8)
        return s["q"], s["scales"]
    if op == "quantise_weight":
        q, scales = _quantise_blocks(s["w"].float())
        return (q.transpose(1, 2).contiguous(), scales.transpose(1, 2)) if case["transpose"] else (q, scales)
    if op == "linear8":
        return _linear8(s, case)
    if op == "norm":
        return _norm(s, case)
    if op == "norm_grad":
        return _norm_grad(s, case)
    return _adamw(s, case)


# ---------------------------------------------------------------- what a pass cannot do without
def _flops(case):
    op = case["op"]
    if op == "linear8":
        return 2 * case["rows"] * case["in"] * case["out"]
    if op == "quantise":
        return 4 * case["rows"] * case["features"]
    if op == "quantise_weight":
        return 3 * case["groups"] * case["out"] * case["in"]
    if op in ("norm", "norm_grad"):
        return case["tokens"] * case["features"] * (10 if op == "norm" else 24)
    return 14 * _parameters(case)


def work(case):
    op, es = case["op"], BYTES[case["dtype"]]
    if op == "quantise":
        n, h = case["rows"], case["features"]
        b = n * h * es * (2 if case["act"] in GATED else 1) + n * h + n * _blocks(h)
    elif op == "quantise_weight":
        n = case["groups"] * case["out"] * case["in"]
        b = n * (es + 1) + case["groups"] * _blocks(case["out"]) * _blocks(case["in"])
    elif op == "linear8":
        n, groups, ki, mo = case["rows"], case["groups"], case["in"], case["out"]
        # groups that have rows (their weights are read)
        full = groups * (1 - (1 - 1 / groups) ** n) if groups > 1 else 1
        b = n * ki + n * _blocks(ki) + int(full * mo * ki) + n * _out_width(case) * es * (2 if case["residual"] else 1)
        b += n * mo * es if case["save"] else 0
    elif op == "norm":
        n, h = case["tokens"], case["features"]
        b = n * h * es * (3 + case["residual"]) + (n * (h + _blocks(h)) if case["q"] else 0)
    elif op == "norm_grad":
        b = case["tokens"] * case["features"] * es * 6
    else:
        # bfloat16 parameters are written, their binary32 masters read and written
        dear = case["layers"] * 3 * case["experts"] * case["ffn"] * case["hidden"]
        n = _parameters(case)
        b = n * (8 + (4 if case["grad"] == "f32" else 2) + case["bits"] // 2) + (2 * dear if case["dtype"] == "bf16" else 0)
        b += n // 32 if case["bits"] == 8 else 0
    return {"bytes": b, "flops": _flops(case)}


# ---------------------------------------------------------------- in 64 bits, from the definitions
def _act64(a, act):
    if act in GATED:
        h = a.shape[-1] // 2
        return _act64(a[..., :h], "silu" if act == "swiglu" else "gelu") * a[..., h:]
    if act == "relu":
        return a.clamp(min=0)
    if act == "gelu":
        return a * (0.5 * torch.special.erfc(-a / math.sqrt(2.0)))
    return a * torch.sigmoid(a) if act == "silu" else a


def _two64(e):
    """2^e, by its bits: powers that a device computes may be a unit off, and a tie is none then."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _codes64(x, amax):
    """(x / s to the nearest e4m3 value, ties to even; s) with s the least power of two that brings amax to 448 or below."""
    frac, e = torch.frexp(amax)  # amax = frac * 2^e, 0.5 <= frac < 1
    e = torch.where(amax > 0, e - 9 + (frac > 0.875).int(), torch.full_like(e, -126)).clamp(min=-126)
    s = _two64(e)
    y = x / s
    step = _two64(torch.frexp(y)[1].clamp(min=-5) - 4)
    return torch.round(y / step) * step, s


def _rows64(x):
    parts = [_codes64(p, p.abs().amax(1, keepdim=True)) for p in x.split(BLOCK, 1)]
    return torch.cat([q for q, _ in parts], 1), torch.cat([s for _, s in parts], 1)


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "quantise":
        n, h = case["rows"], case["features"]
        q, scales = s["q"].double(), s["scales"].double()
        q[:n], scales[:n] = _rows64(_act64(s["x"][:n].double(), case["act"]))
        return q, scales
    if op == "quantise_weight":
        qs, cs = [], []
        for w in s["w"]:
            strips = w.double().split(BLOCK, 0)
            done = [[_codes64(p, p.abs().max()) for p in strip.split(BLOCK, 1)] for strip in strips]
            qs.append(torch.cat([torch.cat([q for q, _ in row], 1) for row in done]))
            cs.append(torch.stack([torch.stack([c for _, c in row]) for row in done]))
        q, c = torch.stack(qs), torch.stack(cs)
        return (q.transpose(1, 2).contiguous(), c.transpose(1, 2).contiguous()) if case["transpose"] else (q, c)
    if op == "linear8":
        cuts, ki = s["bounds"], case["in"]
        ys, zs = [], []
        of_k = torch.arange(ki, device="cuda") // BLOCK
        of_o = torch.arange(case["out"], device="cuda") // BLOCK
        for i in range(case["groups"]):
            lo, hi = cuts[i], cuts[i + 1]
            x = s["x"][lo:hi].double() * s["x_scales"][lo:hi].double()[:, of_k]
            w = s["w"][i].double() * s["w_scales"][i].double()[of_o][:, of_k]
            z = torch.matmul(x, w.transpose(0, 1)) + (s["b"][i].double() if s["b"] is not None else 0)
            zs.append(z)
            ys.append(_act64(z, case["act"]))
        y = torch.cat(ys)
        if s["residual"] is not None:
            y = y + s["residual"].double()
        return (y, torch.cat(zs)) if case["save"] else y
    if op == "norm":
        y = s["y"].double()
        u = y if s["post"] is None else s["post"].double() * y / torch.sqrt(y.square().mean(1, keepdim=True) + EPS)
        r = s["scale"] * (u if s["gate"] is None else s["gate"].double()[:, None] * u)
        r = r if s["residual"] is None else s["residual"].double() + r
        h = s["weight"].double() * r / torch.sqrt(r.square().mean(1, keepdim=True) + EPS)
        return (h, r) + (_rows64(h) if case["q"] else ())
    if op == "norm_grad":
        return _exact_norm_grad(s)
    return _exact_adamw(case, s)


def _exact_norm_grad(s):
    r, dh, w = s["r"].double(), s["dh"].double(), s["weight"].double()
    n = r.shape[1]

    def back(x, d, weight):
        # x / d with d = sqrt(mean x^2 + eps): the quotient's derivative
        den = torch.sqrt(x.square().sum(1, keepdim=True) / n + EPS)
        t = weight[None] * d
        return t / den - x * (t * x).sum(1, keepdim=True) / (n * den ** 3), (d * x / den).sum(0), x / den

    dr, dweight, _ = back(r, dh, w)
    dr = dr + s["dr"].double()
    y = s["y"].double()
    g = s["scale"] * (dr if s["gate"] is None else dr * s["gate"].double()[:, None])
    out = [dr, g]
    u = y
    dpost = None
    if s["post"] is not None:
        out[1], dpost, unit = back(y, g, s["post"].double())
        u = s["post"].double() * unit
    if s["gate"] is not None:
        out.append(s["scale"] * torch.linalg.vecdot(dr, u))
    out.append(dweight)
    return tuple(out + ([] if dpost is None else [dpost]))


def _exact_adamw(case, s):
    t = 41
    params, masters, ms, vs = [], [], [], []
    eight = case["bits"] == 8
    at = 0
    for p, w, g, n in zip(s["params"], s["masters"], s["grads"], s["sizes"]):
        end = at + _padded(n)
        m, v = s["m"][at:end].double(), s["v"][at:end].double()
        if eight:
            m = (m.view(-1, BLOCK) * s["m_scales"][at // BLOCK:end // BLOCK].double()[:, None]).view(-1)
            v = (v.view(-1, BLOCK) * s["v_scales"][at // BLOCK:end // BLOCK].double()[:, None]).view(-1)
        g = g.double().reshape(-1)
        m[:n] = BETA1 * m[:n] + (1 - BETA1) * g
        v[:n] = BETA2 * v[:n] + (1 - BETA2) * g.square()
        x = (p if w is None else w).double().reshape(-1)
        x = x - LR * DECAY * x - LR * (m[:n] / (1 - BETA1 ** t)) / ((v[:n] / (1 - BETA2 ** t)).sqrt() + ADAM_EPS)
        params.append(x)
        if w is not None:
            masters.append(x)
        ms.append(m)
        vs.append(v)
        at = end
    # states in 8 bits are rounded at random: 64 bits say nothing of them
    return params, masters, None if eight else torch.cat(ms), None if eight else torch.cat(vs), None, None, None
