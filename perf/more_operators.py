"""The operators of a feed-forward sublayer in few bits, as measured: microscaled quantisation, norms with an 8-bit output, dense layer and
gated projections of microscaled operands, the norm of all gradients and their clipping.

Microscaled: elements e4m3 or e2m1, one power of two for each 32 neighbours of a row (OCP Microscaling Formats 1.0).  `run` computes in
elementary torch operations in float32 (`own` false) or through the framework's calls (`own` true); what is held in 8 or 4 bits is
returned as the values it stands for.  `exact` states the same results in float64 from the definitions.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
EPS = 1e-6
GELU_C, GELU_A = math.sqrt(2.0 / math.pi), 0.044715
# format: exponent of the largest element, smallest exponent, bits behind the binary point, largest element
FORMATS = {"e4m3": (8, -6, 3, 448.0), "e2m1": (2, 0, 1, 6.0)}


# ---------------------------------------------------------------------------------------------------- cases
def _quantize(name, dtype, rows, cols, fmt, pad):
    return {"name": name, "op": "quantize", "dtype": dtype, "rows": rows, "cols": cols, "fmt": fmt, "pad": pad}


def _norm(name, dtype, rows, cols, kind, post, alpha, shift):
    return {"name": name, "op": "norm", "dtype": dtype, "rows": rows, "cols": cols, "kind": kind, "post": post, "alpha": alpha, "shift": shift}


def _linear(name, dtype, rows, inner, outer, x, w, act, bias, residual, norm, train):
    return {"name": name, "op": "linear", "dtype": dtype, "rows": rows, "inner": inner, "outer": outer, "x": x, "w": w, "act": act, "bias": bias,
            "residual": residual, "norm": norm, "train": train}


def _gated(name, dtype, rows, inner, outer, x, w, act, norm, down):
    return {"name": name, "op": "gated", "dtype": dtype, "rows": rows, "inner": inner, "outer": outer, "x": x, "w": w, "act": act, "norm": norm,
            "down": down}


def _clip(name, dtype, layers, width, inner, mixed, max_norm):
    return {"name": name, "op": "clip", "dtype": dtype, "layers": layers, "width": width, "inner": inner, "mixed": mixed, "max_norm": max_norm}


def listed():
    return [
        # master weights of odd sizes, a slice of a wider buffer, to 4 bits after an update
        _quantize("quantize-odd", "f32", 333, 1011, "e2m1", 3),
        # a batch of activations to 8 bits, with the values for the backward pass
        _quantize("quantize-train", "bf16", 8192, 4096, "e4m3", 0),
        # the glue between two blocks for one generated token
        _norm("norm-token", "bf16", 1, 4096, "rms", True, 1.0, False),
        # the same for a prompt or a training batch: residual, norm, 8 bits
        _norm("norm-prompt", "bf16", 8192, 4096, "rms", False, 1.0, False),
        # one token: norm in 8 bits and a projection with 4-bit weights back to the residual stream
        _linear("linear-token", "bf16", 1, 4096, 4096, "e4m3", "e2m1", "none", True, True, True, False),
        # a ragged batch in 8 bits, widths that are no multiple of a block
        _linear("linear-ragged", "f16", 1000, 4100, 1010, "e4m3", "e4m3", "relu", True, False, False, False),
        # a prompt with weights and activations in 4 bits
        _linear("linear-prompt", "bf16", 8192, 4096, 8192, "e2m1", "e2m1", "none", False, True, False, False),
        # a training step with 8-bit operands forward and the straight-through gradients
        _linear("linear-train", "bf16", 4096, 2048, 4096, "e4m3", "e4m3", "gelu", True, False, False, True),
        # a few dozen sequences decoded together through both projections of a gated block
        _gated("gated-batch", "f16", 48, 2048, 5500, "e4m3", "e2m1", "gelu_tanh", True, False),
        # a whole gated sublayer for a prompt: norm, both projections, their product in 8 bits, the projection back
        _gated("sublayer-prompt", "bf16", 4096, 4096, 8192, "e4m3", "e2m1", "silu", True, True),
        # the gradients of one odd-sized layer
        _clip("clip-layer", "f32", 1, 333, 1011, False, 1.0),
        # the gradients of a model: matrices in 16 bits, vectors in 32
        _clip("clip-model", "bf16", 7, 2048, 8192, True, 1.0),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    n = _log(rng, low, high)
    return n if rng.random() < 0.3 else max(low, n // 32 * 32)


def draw(rng):
    op = rng.choice(("quantize", "norm", "linear", "gated", "clip"))
    half = rng.choice(("bf16", "f16"))
    x, w = rng.choice((("e4m3", "e4m3"), ("e4m3", "e2m1"), ("e2m1", "e2m1")))
    if op == "quantize":
        case = _quantize("", rng.choice(("bf16", "f16", "f32")), _log(rng, 1, 8192), _width(rng, 32, 8192), rng.choice(("e4m3", "e2m1")),
                         rng.choice((0, 0, 3, 8)))
    elif op == "norm":
        case = _norm("", half, _log(rng, 1, 8192), _width(rng, 64, 8192), rng.choice(("rms", "layer")), rng.random() < 0.5, rng.choice((1.0, 0.5)),
                     rng.random() < 0.3)
    elif op == "linear":
        train = rng.random() < 0.2
        case = _linear("", half, _log(rng, 1, 4096), _width(rng, 64, 4096 if train else 8192), _width(rng, 64, 4096 if train else 8192), x, w,
                       rng.choice(ACTS), rng.random() < 0.5, rng.random() < 0.5, False, train)
        case["norm"] = case["x"] == "e4m3" and not case["train"] and rng.random() < 0.5
    elif op == "gated":
        case = _gated("", half, _log(rng, 1, 4096), _width(rng, 64, 4096), _width(rng, 64, 8192), x, w, rng.choice(ACTS[1:]), False, False)
        case["norm"], case["down"] = case["x"] == "e4m3" and rng.random() < 0.5, case["x"] == "e4m3" and rng.random() < 0.5
    else:
        case = _clip("", rng.choice(("bf16", "f16", "f32")), rng.randint(1, 7), _log(rng, 64, 1024), _log(rng, 64, 8192), rng.random() < 0.5,
                     rng.choice((0.5, 1.0, 1e9)))
    del case["name"]
    return case


def _mx_bytes(fmt, n):
    return n * (0.5 if fmt == "e2m1" else 1.0) + n / 32


def work(case):
    e, op = (4 if case["dtype"] == "f32" else 2), case["op"]
    if op == "clip":
        d, f, n = case["width"], case["inner"], case["layers"]
        v = 4 if case["mixed"] else e
        return {"bytes": 2 * n * (e * 3 * d * f + v * (4 * d + f)), "flops": 3 * n * 3 * d * f}
    m = case["rows"]
    if op == "quantize":
        return {"bytes": m * case["cols"] * 2 * e + _mx_bytes(case["fmt"], m * case["cols"]), "flops": 3 * m * case["cols"]}
    if op == "norm":
        return {"bytes": m * case["cols"] * 4 * e + _mx_bytes("e4m3", m * case["cols"]), "flops": 12 * m * case["cols"]}
    k, n = case["inner"], case["outer"]
    inputs = e * m * k * (3 if case["norm"] else 1)                       # two rows in and the stream out, or x
    if op == "gated":
        weights, out = _mx_bytes(case["w"], 2 * n * k), e * m * n
        if case["down"]:
            weights, out = weights + _mx_bytes(case["w"], n * k), 2 * e * m * k
        return {"bytes": inputs + weights + out, "flops": (6 if case["down"] else 4) * m * n * k}
    if case["train"]:                                                     # x, W, dy, bias; y, dx, dW, db
        return {"bytes": e * (2 * m * k + 2 * n * k + m * n * (2 + case["residual"]) + 2 * n * case["bias"]), "flops": 6 * m * n * k}
    return {"bytes": inputs + _mx_bytes(case["w"], n * k) + e * (m * n * (1 + case["residual"]) + n * case["bias"]), "flops": 2 * m * n * k}


# ---------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    dtype = DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, shift=0.0, to=dtype):
        return torch.empty(*shape, device="cuda").normal_(shift, scale, generator=gen).to(to)

    def rows_of(m, d, scale):                         # channels of unlike sizes, as a block's inputs have them
        return (torch.empty(m, d, device="cuda").normal_(0.0, scale, generator=gen) * torch.exp(normal(d, scale=0.7, to=torch.float32))).to(dtype)

    s = {"case": dict(case), "kept": {}}
    if case["op"] == "clip":
        d, f, wide = case["width"], case["inner"], torch.float32 if case["mixed"] else dtype
        shapes = [((f, d), dtype), ((f, d), dtype), ((d, f), dtype), ((d,), wide), ((d,), wide), ((d,), wide), ((d,), wide), ((f,), wide)]
        s["grads"] = [normal(*shape, scale=0.02, to=t) for _ in range(case["layers"]) for shape, t in shapes]
        return s
    m = case["rows"]
    if case["op"] == "quantize":
        s["x"] = rows_of(m, case["cols"] + case["pad"], 1.0)[:, :case["cols"]]
        return s
    if case["op"] == "norm" or case["norm"]:
        d = case["cols"] if case["op"] == "norm" else case["inner"]
        s["stream"], s["block"] = rows_of(m, d, 2.0), normal(m, d, scale=0.5, shift=0.1)
        s["pre_w"] = normal(d, scale=0.1, shift=1.0)
        s["pre_c"] = normal(d, scale=0.1) if case.get("shift") else None
        s["post_w"] = normal(d, scale=0.1, shift=1.0) if case.get("post") else None
    else:
        s["x"] = rows_of(m, case["inner"], 1.0)
    if case["op"] == "linear":
        k, n = case["inner"], case["outer"]
        s["W"] = normal(n, k, scale=k ** -0.5)
        s["bias"] = normal(n, scale=0.5) if case["bias"] else None
        s["residual"] = normal(m, n, scale=2.0) if case["residual"] else None
        s["dy"] = normal(m, n, scale=0.1) if case["train"] else None
    elif case["op"] == "gated":
        k, n = case["inner"], case["outer"]
        s["Wg"], s["Wu"] = normal(n, k, scale=k ** -0.5), normal(n, k, scale=k ** -0.5)
        s["Wd"] = normal(k, n, scale=n ** -0.5) if case["down"] else None
    return s


# ---------------------------------------------------------------------------------------------------- plain forms
def _pow2(e):
    """2 ^ e for whole e of -149 .. 127, in float32."""
    half = torch.div(e, 2, rounding_mode="floor")
    return torch.ldexp(torch.ones_like(e, dtype=torch.float32), half) * torch.ldexp(torch.ones_like(e, dtype=torch.float32), e - half)


def _mx(v, fmt):
    """The values that the microscaled form of the float32 rows v stands for."""
    emax, emin, digits, most = FORMATS[fmt]
    m, k = v.shape
    b = torch.nn.functional.pad(v, (0, -k % 32)).reshape(m, -1, 32)
    amax = b.abs().amax(2, keepdim=True)
    shared = torch.where(amax > 0, torch.frexp(amax)[1] - 1 - emax, -127).clamp(-127, 127)
    u = b * _pow2(-(shared // 2)) * _pow2(shared // 2 - shared)
    step = _pow2((torch.frexp(u)[1] - 1).clamp_min(emin) - digits)
    q = (torch.round(u / step) * step).clamp(-most, most) * _pow2(shared // 2) * _pow2(shared - shared // 2)
    return torch.where(torch.isfinite(amax), q, math.nan).reshape(m, -1)[:, :k]


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(GELU_C * (z + GELU_A * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        t = torch.tanh(GELU_C * (z + GELU_A * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * GELU_C * (1 + 3 * GELU_A * z * z)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def _norm_rows(v, w, c, kind):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    v = v / torch.sqrt((v * v).mean(1, keepdim=True) + EPS) * w.float()
    return v if c is None else v + c.float()


def _stream_plain(s):
    """The residual stream and its norm, in float32."""
    c = s["case"]
    kind = c.get("kind", "rms")
    p = s["block"].float()
    if s["post_w"] is not None:
        p = _norm_rows(p, s["post_w"], None, kind)
    stream = c.get("alpha", 1.0) * s["stream"].float() + p
    return stream, _norm_rows(stream, s["pre_w"], s["pre_c"], kind)


def _quantize_plain(s):
    return {"values": _mx(s["x"].float(), s["case"]["fmt"]).to(DTYPES[s["case"]["dtype"]])}


def _norm_plain(s):
    dtype = DTYPES[s["case"]["dtype"]]
    stream, normed = _stream_plain(s)
    return {"stream": stream.to(dtype), "values": _mx(normed, "e4m3").to(dtype)}


def _inputs_plain(s):
    """The product's left operand, and the stream where a norm comes first."""
    if not s["case"]["norm"]:
        return {}, _mx(s["x"].float(), s["case"]["x"])
    stream, normed = _stream_plain(s)
    return {"stream": stream.to(DTYPES[s["case"]["dtype"]])}, _mx(normed, s["case"]["x"])


def _linear_plain(s):
    c, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    out, x = _inputs_plain(s)
    w = _mx(s["W"].float(), c["w"])
    z = x @ w.T
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = s["residual"].float() + y
    out["y"] = y.to(dtype)
    if c["train"]:
        dz = s["dy"].float() * _act_slope(z, c["act"])
        out |= {"dx": (dz @ w).to(dtype), "dW": (dz.T @ x).to(dtype)}
        if s["bias"] is not None:
            out["db"] = dz.sum(0).to(dtype)
    return out


def _gated_plain(s):
    c, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    out, x = _inputs_plain(s)
    h = _act(x @ _mx(s["Wg"].float(), c["w"]).T, c["act"]) * (x @ _mx(s["Wu"].float(), c["w"]).T)
    if not c["down"]:
        return out | {"h": h.to(dtype)}
    return out | {"y": (_mx(h, c["x"]) @ _mx(s["Wd"].float(), c["w"]).T).to(dtype)}


def _clip_plain(s):
    norm = torch.sqrt(torch.stack([g.double().square().sum() for g in s["grads"]]).sum())
    factor = torch.clamp(s["case"]["max_norm"] / (norm + EPS), max=1.0).float()
    return {"norm": norm.float(), "grads": [(g.float() * factor).to(g.dtype) for g in s["grads"]]}


# ---------------------------------------------------------------------------------------------------- the framework's calls
_held = {}


def _context(need=0):
    """The program's context, with a workspace of at least `need` bytes lent to it."""
    if "ctx" not in _held:
        from paper_1602_02830_b200 import binding
        _held["ctx"] = binding.Context(torch.cuda.current_device())
    if need > _held.get("bytes", 0):
        _held["space"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        _held["bytes"] = need
        _held["ctx"].set_workspace(_held["space"])
    return _held["ctx"]


def _norm_handle(ctx, s):
    c = s["case"]
    return ctx.make_block_norm(s["stream"].shape[1], DTYPES[c["dtype"]], kind=c.get("kind", "rms"), eps=EPS, alpha=c.get("alpha", 1.0),
                               post=s["post_w"] is not None, post_weight=s["post_w"], pre_weight=s["pre_w"], pre_shift=s["pre_c"])


def _quantize_own(s):
    c, kept, ctx = s["case"], s["kept"], _context()
    if not kept:
        kept["q"] = ctx.make_mx(c["rows"], c["cols"], c["fmt"])
    values = ctx.empty(c["rows"], c["cols"], dtype=DTYPES[c["dtype"]])
    ctx.mx_quantize(s["x"], out=kept["q"], values=values)
    return {"values": values}


def _norm_own(s):
    c, kept, ctx = s["case"], s["kept"], _context()
    if not kept:
        kept["norm"] = _norm_handle(ctx, s)
        kept["q"] = ctx.make_mx(c["rows"], c["cols"], "e4m3")
    values = ctx.empty(c["rows"], c["cols"], dtype=DTYPES[c["dtype"]])
    stream, _ = ctx.block_norm_mx(kept["norm"], s["stream"], s["block"], out=kept["q"], values=values)
    return {"stream": stream, "values": values}


def _inputs_own(ctx, s):
    c, kept = s["case"], s["kept"]
    if "q" not in kept:
        kept["q"] = ctx.make_mx(c["rows"], c["inner"], c["x"])
        kept["norm"] = _norm_handle(ctx, s) if c["norm"] else None
    if not c["norm"]:
        ctx.mx_quantize(s["x"], out=kept["q"])
        return {}, kept["q"]
    stream, _ = ctx.block_norm_mx(kept["norm"], s["stream"], s["block"], out=kept["q"])
    return {"stream": stream}, kept["q"]


def _linear_own(s):
    c, kept, dtype, ctx = s["case"], s["kept"], DTYPES[s["case"]["dtype"]], _context()
    if not c["train"]:
        if "layer" not in kept:                       # the weights, quantised and laid out once
            kept["layer"] = ctx.make_mx_linear(ctx.mx_quantize(s["W"], c["w"]), s["bias"], c["act"], dtype=dtype)
        out, q = _inputs_own(ctx, s)
        return out | {"y": ctx.mx_linear(kept["layer"], q, s["residual"])}
    if "layer" not in kept:                           # buffers and handles; the weights change from step to step
        kept["q"], kept["Wq"] = ctx.make_mx(c["rows"], c["inner"], c["x"]), ctx.make_mx(c["outer"], c["inner"], c["w"])
        kept["x"], kept["W"] = torch.empty_like(s["x"]), torch.empty_like(s["W"])
        kept["layer"] = ctx.make_mx_linear(kept["Wq"], s["bias"], c["act"], dtype=dtype)
        kept["back"] = ctx.make_linear(kept["W"], s["bias"], c["act"])
        kept["need"] = ctx.linear_workspace_bytes(kept["back"], kept["x"], backward=True)
    ctx = _context(kept["need"])
    ctx.mx_quantize(s["W"], out=kept["Wq"], values=kept["W"])
    ctx.mx_quantize(s["x"], out=kept["q"], values=kept["x"])
    pre = ctx.empty(c["rows"], c["outer"], dtype=torch.float32) if c["act"] != "none" else None
    out = {"y": ctx.mx_linear(kept["layer"], kept["q"], s["residual"], pre=pre)}
    out["dx"], out["dW"], db = ctx.linear_backward(kept["back"], s["dy"], kept["x"], pre=pre)
    return out if db is None else out | {"db": db}


def _gated_own(s):
    c, kept, dtype, ctx = s["case"], s["kept"], DTYPES[s["case"]["dtype"]], _context()
    if "layer" not in kept:
        kept["layer"] = ctx.make_mx_gated(ctx.mx_quantize(s["Wg"], c["w"]), ctx.mx_quantize(s["Wu"], c["w"]), c["act"], dtype=dtype)
        if c["down"]:
            kept["h"] = ctx.make_mx(c["rows"], c["outer"], c["x"])
            kept["back"] = ctx.make_mx_linear(ctx.mx_quantize(s["Wd"], c["w"]), dtype=dtype)
    out, q = _inputs_own(ctx, s)
    if not c["down"]:
        return out | {"h": ctx.mx_gated(kept["layer"], q)}
    return out | {"y": ctx.mx_linear(kept["back"], ctx.mx_gated(kept["layer"], q, out=kept["h"]))}


def _clip_own(s):
    kept, ctx = s["kept"], _context()
    if not kept:
        kept["out"] = [torch.empty_like(g) for g in s["grads"]]
        kept["set"] = ctx.make_gradients(s["grads"], out=kept["out"])
        kept["need"] = ctx.clip_workspace_bytes(kept["set"])
    norm = _context(kept["need"]).clip_gradients(kept["set"], s["case"]["max_norm"], eps=EPS)
    return {"norm": norm, "grads": kept["out"]}


def run(state):
    op = state["case"]["op"]
    if own:
        return {"quantize": _quantize_own, "norm": _norm_own, "linear": _linear_own, "gated": _gated_own, "clip": _clip_own}[op](state)
    return {"quantize": _quantize_plain, "norm": _norm_plain, "linear": _linear_plain, "gated": _gated_plain, "clip": _clip_plain}[op](state)


# ---------------------------------------------------------------------------------------------------- float64
def _elements(fmt):
    """All elements >= 0 of a format, in the order of their codes."""
    bits, bias = (3, 7) if fmt == "e4m3" else (1, 1)
    codes = range(127 if fmt == "e4m3" else 8)
    return torch.tensor([(c & (1 << bits) - 1) * 2.0 ** (1 - bias - bits) if c >> bits == 0 else
                         (1 + (c & (1 << bits) - 1) / (1 << bits)) * 2.0 ** ((c >> bits) - bias) for c in codes], dtype=torch.float64, device="cuda")


def _mx64(v, fmt):
    """The nearest element to each value, the even code on a tie; the scale is the largest power of two not above the block's largest value,
    taken by the format's own exponent."""
    table = _elements(fmt)
    m, k = v.shape
    blocks = torch.cat([v, v.new_zeros(m, -k % 32)], 1).unflatten(1, (-1, 32))
    top = blocks.abs().max(2, keepdim=True).values
    guess = torch.floor(torch.log2(top.clamp_min(1e-300)))
    guess = guess - (torch.exp2(guess) > top).double() + (torch.exp2(guess + 1) <= top).double()
    scale = torch.exp2((guess - (8 if fmt == "e4m3" else 2)).clamp(-127, 127))
    size = blocks.abs() / scale
    high = torch.searchsorted(table, size).clamp_max(len(table) - 1)
    low = (high - 1).clamp_min(0)
    up, down = table[high] - size, size - table[low]
    code = torch.where((up < down) | ((up == down) & (high % 2 == 0)), high, low)
    return (torch.sign(blocks) * table[code] * scale).flatten(1)[:, :k]


def _act64(z, act):
    fn = torch.nn.functional
    return {"none": lambda: z, "relu": lambda: fn.relu(z), "gelu": lambda: fn.gelu(z), "silu": lambda: fn.silu(z),
            "gelu_tanh": lambda: fn.gelu(z, approximate="tanh")}[act]()


def _norm64(v, w, c, kind):
    mean = v.mean(1, keepdim=True) if kind == "layer" else 0.0
    y = (v - mean) / ((v - mean).pow(2).mean(1, keepdim=True) + EPS).sqrt() * w.double()
    return y if c is None else y + c.double()


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "clip":
        # the root of the sum by numbers of 64 bits, largest first out of the square
        top = max(float(g.abs().max()) for g in s["grads"])
        norm = top * math.sqrt(math.fsum(float((g.double() / top).pow(2).sum()) for g in s["grads"]))
        factor = min(1.0, case["max_norm"] / (norm + EPS))
        return {"norm": torch.tensor(norm, dtype=torch.float64, device="cuda"), "grads": [g.double() * factor for g in s["grads"]]}
    if op == "quantize":
        return {"values": _mx64(s["x"].double(), case["fmt"])}
    outs = {}
    if op == "norm" or case["norm"]:
        kind, p = case.get("kind", "rms"), s["block"].double()
        if s["post_w"] is not None:
            p = _norm64(p, s["post_w"], None, kind)
        outs["stream"] = case.get("alpha", 1.0) * s["stream"].double() + p
        x = _norm64(outs["stream"], s["pre_w"], s["pre_c"], kind)
    else:
        x = s["x"].double()
    if op == "norm":
        return outs | {"values": _mx64(x, "e4m3")}
    x = _mx64(x, case["x"])
    if op == "gated":
        h = _act64(x @ _mx64(s["Wg"].double(), case["w"]).T, case["act"]) * (x @ _mx64(s["Wu"].double(), case["w"]).T)
        return outs | ({"y": _mx64(h, case["x"]) @ _mx64(s["Wd"].double(), case["w"]).T} if case["down"] else {"h": h})
    # gradients by differentiation at the rounded operands, straight through the rounding
    x, w = x.requires_grad_(case["train"]), _mx64(s["W"].double(), case["w"]).requires_grad_(case["train"])
    b = None if s["bias"] is None else s["bias"].double().requires_grad_(case["train"])
    y = _act64(x @ w.T if b is None else torch.addmm(b, x, w.T), case["act"])
    if s["residual"] is not None:
        y = y + s["residual"].double()
    outs["y"] = y.detach()
    if case["train"]:
        wanted = {"dx": x, "dW": w} | ({} if b is None else {"db": b})
        outs |= dict(zip(wanted, torch.autograd.grad(y, list(wanted.values()), s["dy"].double())))
    return outs
