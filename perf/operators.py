"""The operators of a real-valued feed-forward sublayer, as measured: dense layer with its epilogue, gated projections,
norms around a block, dropout without a stored mask.

`run` computes them in elementary torch operations in float32 (`own` false) or through the framework's calls (`own` true);
`exact` states the same results in float64 from the definitions, gradients by differentiation.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu", "sigmoid", "htanh")
GLU_ACTS = ("silu", "gelu", "gelu_tanh", "sigmoid", "relu")
EPS = 1e-6
GELU_C, GELU_A = math.sqrt(2.0 / math.pi), 0.044715


# ---------------------------------------------------------------------------------------------------- cases
def _linear(name, dtype, rows, inner, outer, act, bias, residual, pad, train):
    return {"name": name, "op": "linear", "dtype": dtype, "rows": rows, "inner": inner, "outer": outer, "act": act, "bias": bias,
            "residual": residual, "pad": pad, "train": train}


def _gated(name, dtype, rows, inner, outer, act, train):
    return {"name": name, "op": "gated", "dtype": dtype, "rows": rows, "inner": inner, "outer": outer, "act": act, "train": train}


def _norm(name, dtype, rows, cols, kind, post, gates, alpha, shift, train):
    return {"name": name, "op": "norm", "dtype": dtype, "rows": rows, "cols": cols, "kind": kind, "post": post, "gates": gates,
            "alpha": alpha, "shift": shift, "train": train}


def _dropout(name, dtype, rows, cols, p, residual, train):
    return {"name": name, "op": "dropout", "dtype": dtype, "rows": rows, "cols": cols, "p": p, "residual": residual, "train": train}


def listed():
    return [
        # one generated token through a square projection that adds to the residual stream: latency and weight bytes
        _linear("linear-token", "bf16", 1, 4096, 4096, "none", True, True, 0, False),
        # a ragged batch: row pitches that are not whole 16-byte groups, inputs that are a slice of a wider buffer
        _linear("linear-ragged", "f16", 1000, 4100, 1010, "relu", True, False, 3, False),
        # the projection back to the residual stream for a prompt
        _linear("linear-prompt", "bf16", 2048, 8192, 4096, "none", False, True, 0, False),
        # a dense layer of 4096 units in training: forward, all gradients
        _linear("linear-train", "bf16", 8192, 4096, 4096, "gelu", True, True, 0, True),
        # one generated token through both projections of a gated block
        _gated("gated-token", "bf16", 1, 4096, 8192, "silu", False),
        # a few dozen sequences decoded together, a width that is no multiple of any tile
        _gated("gated-batch", "f16", 48, 2048, 5500, "gelu_tanh", False),
        # the gated block in training: forward, all gradients
        _gated("gated-train", "bf16", 8192, 4096, 8192, "silu", True),
        # the glue between two blocks for one token
        _norm("norm-token", "bf16", 1, 4096, "rms", True, 1, 1.0, False, False),
        # layer norm with shifts of an odd width in float32, no norm after the block, gates per sequence, in training
        _norm("norm-odd", "f32", 1000, 1011, "layer", False, 8, 0.5, True, True),
        # norm after the block, channel gate, residual, norm before the next block, in training
        _norm("norm-train", "bf16", 8192, 4096, "rms", True, 1, 1.0, False, True),
        # an odd-sized activation in float32, forward and backward
        _dropout("dropout-odd", "f32", 333, 1011, 0.5, False, True),
        # a block's output dropped and added to the residual stream, forward and backward
        _dropout("dropout-train", "bf16", 16384, 4096, 0.1, True, True),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def _width(rng, low, high):
    n = _log(rng, low, high)
    return n if rng.random() < 0.3 else max(low, n // 8 * 8)


def draw(rng):
    op = rng.choice(("linear", "gated", "norm", "dropout"))
    train = rng.random() < 0.5
    if op == "linear":
        case = _linear("", rng.choice(("bf16", "f16")), _log(rng, 1, 8192), _width(rng, 64, 8192), _width(rng, 64, 8192),
                       rng.choice(ACTS), rng.random() < 0.5, rng.random() < 0.5, rng.choice((0, 0, 3, 8)), train)
    elif op == "gated":
        case = _gated("", rng.choice(("bf16", "f16")), _log(rng, 1, 8192), _width(rng, 64, 4096), _width(rng, 64, 8192),
                      rng.choice(GLU_ACTS), train)
    elif op == "norm":
        case = _norm("", rng.choice(("bf16", "f16", "f32")), _log(rng, 1, 8192), _width(rng, 64, 8192), rng.choice(("rms", "layer")),
                     rng.random() < 0.5, rng.choice((0, 1, 4)), rng.choice((1.0, 0.5)), rng.random() < 0.5, train)
    else:
        case = _dropout("", rng.choice(("bf16", "f16", "f32")), _log(rng, 1, 16384), _width(rng, 64, 4096), rng.choice((0.1, 0.2, 0.5)),
                        rng.random() < 0.5, train)
    del case["name"]
    return case


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    m = case["rows"]
    if case["op"] == "linear":
        k, n, t = case["inner"], case["outer"], case["train"]
        elements = m * k + n * k + m * n * (1 + case["residual"]) + n * case["bias"]
        if t:
            elements += m * n + m * k + n * k + n * case["bias"]
        return {"bytes": e * elements, "flops": (6 if t else 2) * m * n * k}
    if case["op"] == "gated":
        d, f, t = case["inner"], case["outer"], case["train"]
        return {"bytes": e * (2 if t else 1) * (m * d + 2 * f * d + m * f), "flops": (12 if t else 4) * m * d * f}
    d = case["cols"]
    if case["op"] == "norm":
        return {"bytes": e * m * d * (8 if case["train"] else 4), "flops": m * d * (40 if case["train"] else 14)}
    moved = 2 + case["residual"] + (2 if case["train"] else 0)
    return {"bytes": e * m * d * moved, "flops": 0}


# ---------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    dtype = DTYPES[case["dtype"]]
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, shift=0.0):
        return torch.empty(*shape, device="cuda").normal_(shift, scale, generator=gen).to(dtype)

    s = {"case": dict(case), "kept": {}}
    m = case["rows"]
    if case["op"] in ("linear", "gated"):
        k, n = case["inner"], case["outer"]
        pad = case.get("pad", 0)
        s["x"] = normal(m, k + pad)[:, :k]
        s["dy"] = normal(m, n, scale=0.1) if case["train"] else None
        if case["op"] == "linear":
            s["W"] = normal(n, k, scale=k ** -0.5)
            s["bias"] = normal(n, scale=0.5) if case["bias"] else None
            s["residual"] = normal(m, n, scale=2.0) if case["residual"] else None
        else:
            s["Wg"], s["Wu"] = normal(n, k, scale=k ** -0.5), normal(n, k, scale=k ** -0.5)
        return s
    d = case["cols"]
    s["x"] = normal(m, d, scale=2.0)
    if case["op"] == "norm":
        s["block"] = normal(m, d, scale=0.5, shift=0.1)
        s["pre_w"] = normal(d, scale=0.1, shift=1.0)
        s["pre_c"] = normal(d, scale=0.1) if case["shift"] else None
        s["post_w"] = normal(d, scale=0.1, shift=1.0) if case["post"] else None
        s["post_c"] = normal(d, scale=0.1) if case["post"] and case["shift"] else None
        s["gate"] = normal(case["gates"], d, scale=0.3, shift=0.5) if case["gates"] else None
        s["per_gate"] = -(-m // max(1, case["gates"]))
        s["dstream"] = normal(m, d, scale=0.1) if case["train"] else None
        s["dnormed"] = normal(m, d, scale=0.1) if case["train"] else None
    else:
        s["residual"] = normal(m, d, scale=2.0) if case["residual"] else None
        s["dy"] = normal(m, d, scale=0.1) if case["train"] else None
        s["seed"], s["offset"] = seed * 2654435761 % (1 << 63), seed % 1000
    return s


# ---------------------------------------------------------------------------------------------------- plain forms
def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(GELU_C * (z + GELU_A * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    if act == "htanh":
        return torch.where(z > 1, 1.0, torch.where(z < -1, -1.0, z))
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
    if act == "sigmoid":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 - p)
    if act == "htanh":
        return (z.abs() <= 1).float()
    return torch.ones_like(z)


def _linear_plain(s):
    c, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    x, w = s["x"].float(), s["W"].float()
    z = x @ w.T
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y = _act(z, c["act"])
    if s["residual"] is not None:
        y = s["residual"].float() + y
    out = {"y": y.to(dtype)}
    if c["train"]:
        dz = s["dy"].float() * _act_slope(z, c["act"])
        out |= {"dx": (dz @ w).to(dtype), "dW": (dz.T @ x).to(dtype)}
        if s["bias"] is not None:
            out["db"] = dz.sum(0).to(dtype)
    return out


def _gated_plain(s):
    c, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    x, wg, wu = s["x"].float(), s["Wg"].float(), s["Wu"].float()
    g, u = x @ wg.T, x @ wu.T
    a = _act(g, c["act"])
    out = {"h": (a * u).to(dtype)}
    if c["train"]:
        dh = s["dy"].float()
        dg, du = dh * u * _act_slope(g, c["act"]), dh * a
        out |= {"dx": (dg @ wg + du @ wu).to(dtype), "dWg": (dg.T @ x).to(dtype), "dWu": (du.T @ x).to(dtype)}
    return out


def _norm_rows(v, kind):
    """The normalised rows and the reciprocal deviations."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + EPS)
    return v * r, r


def _norm_rows_back(d, unit, r, kind):
    """The gradient of the rows from that of the normalised rows."""
    inner = d - unit * (d * unit).mean(1, keepdim=True)
    if kind == "layer":
        inner = inner - d.mean(1, keepdim=True)
    return r * inner


def _norm_plain(s):
    c, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    kind = c["kind"]
    x, p = s["x"].float(), s["block"].float()
    m, d = x.shape
    groups = torch.arange(m, device=x.device) // s["per_gate"]
    if c["post"]:
        unit_b, r_b = _norm_rows(p, kind)
        p = unit_b * s["post_w"].float()
        if s["post_c"] is not None:
            p = p + s["post_c"].float()
    gate = s["gate"].float()[groups] if s["gate"] is not None else 1.0
    stream = c["alpha"] * x + gate * p
    unit, r = _norm_rows(stream, kind)
    normed = unit * s["pre_w"].float()
    if s["pre_c"] is not None:
        normed = normed + s["pre_c"].float()
    out = {"stream": stream.to(dtype), "normed": normed.to(dtype)}
    if not c["train"]:
        return out
    dn = s["dnormed"].float()
    total = s["dstream"].float() + _norm_rows_back(dn * s["pre_w"].float(), unit, r, kind)
    out["dx"] = (c["alpha"] * total).to(dtype)
    out["dpre_w"] = (dn * unit).sum(0).to(dtype)
    if s["pre_c"] is not None:
        out["dpre_c"] = dn.sum(0).to(dtype)
    if s["gate"] is not None:
        padded = torch.zeros(c["gates"] * s["per_gate"], d, device=x.device)
        padded[:m] = total * p
        out["dgate"] = padded.reshape(c["gates"], s["per_gate"], d).sum(1).to(dtype)
    dp = gate * total
    if c["post"]:
        out["dpost_w"] = (dp * unit_b).sum(0).to(dtype)
        if s["post_c"] is not None:
            out["dpost_c"] = dp.sum(0).to(dtype)
        dp = _norm_rows_back(dp * s["post_w"].float(), unit_b, r_b, kind)
    out["dblock"] = dp.to(dtype)
    return out


def _kept(shape, p, seed, offset, device):
    """Truth values by Philox4x32-10 (Salmon, Moraes, Dror, Shaw, 2011): counter (element / 4, offset), key seed."""
    low = 0xFFFFFFFF
    n = shape[0] * shape[1]
    group = torch.arange((n + 3) // 4, device=device)
    c0, c1 = group & low, group >> 32
    c2, c3 = torch.full_like(group, offset & low), torch.full_like(group, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57       # 64 bits of the product, whatever the sign
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return (torch.stack((c0, c1, c2, c3), 1).reshape(-1)[:n] >= round(p * 2 ** 32)).reshape(shape)


def _dropout_plain(s):
    c, dtype = s["case"], DTYPES[s["case"]["dtype"]]
    kept = _kept(s["x"].shape, c["p"], s["seed"], s["offset"], s["x"].device)
    scale = 1 / (1 - c["p"])
    y = torch.where(kept, s["x"].float() * scale, 0.0)
    if s["residual"] is not None:
        y = s["residual"].float() + y
    out = {"y": y.to(dtype)}
    if c["train"]:
        out["dx"] = torch.where(kept, s["dy"].float() * scale, 0.0).to(dtype)
    return out


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


def _linear_own(s):
    c, kept = s["case"], s["kept"]
    if not kept:                                      # the layer's handle, made once as a program does
        kept["layer"] = _context().make_linear(s["W"], s["bias"], c["act"])
        kept["need"] = _context().linear_workspace_bytes(kept["layer"], s["x"], backward=c["train"])
    ctx = _context(kept["need"])
    if not c["train"]:
        return {"y": ctx.linear(kept["layer"], s["x"], s["residual"])}
    pre = ctx.empty(c["rows"], c["outer"], dtype=torch.float32) if c["act"] != "none" else None
    out = {"y": ctx.linear(kept["layer"], s["x"], s["residual"], pre=pre)}
    out["dx"], out["dW"], db = ctx.linear_backward(kept["layer"], s["dy"], s["x"], pre=pre)
    if db is not None:
        out["db"] = db
    return out


def _gated_own(s):
    c, kept = s["case"], s["kept"]
    if not kept:
        kept["layer"] = _context().make_gated(s["Wg"], s["Wu"], c["act"])
        kept["need"] = _context().gated_workspace_bytes(kept["layer"], s["x"], backward=c["train"])
    ctx = _context(kept["need"])
    if not c["train"]:
        return {"h": ctx.gated(kept["layer"], s["x"])}
    pre = ctx.empty(2, c["rows"], c["outer"], dtype=torch.float32)
    out = {"h": ctx.gated(kept["layer"], s["x"], pre=pre)}
    out["dx"], out["dWg"], out["dWu"] = ctx.gated_backward(kept["layer"], s["dy"], s["x"], pre=pre)
    return out


def _norm_own(s):
    c, kept = s["case"], s["kept"]
    if not kept:
        kept["norm"] = _context().make_block_norm(
            c["cols"], DTYPES[c["dtype"]], kind=c["kind"], eps=EPS, alpha=c["alpha"], gate=s["gate"], rows_per_gate=s["per_gate"],
            post=c["post"], post_weight=s["post_w"], post_shift=s["post_c"], pre_weight=s["pre_w"], pre_shift=s["pre_c"])
        kept["need"] = _context().block_norm_workspace_bytes(kept["norm"], c["rows"]) if c["train"] else 0
    ctx = _context(kept["need"])
    if not c["train"]:
        stream, normed = ctx.block_norm(kept["norm"], s["x"], s["block"])
        return {"stream": stream, "normed": normed}
    stats = ctx.empty(c["rows"], 4, dtype=torch.float32)
    stream, normed = ctx.block_norm(kept["norm"], s["x"], s["block"], stats=stats)
    back = ctx.block_norm_backward(kept["norm"], s["dstream"], s["dnormed"], s["x"], s["block"], stats)
    names = {"dx": "dx", "dblock": "dblock", "dgate": "dgate", "dpre_weight": "dpre_w", "dpre_shift": "dpre_c",
             "dpost_weight": "dpost_w", "dpost_shift": "dpost_c"}
    return {"stream": stream, "normed": normed} | {names[k]: v for k, v in back.items() if v is not None}


def _dropout_own(s):
    c, ctx = s["case"], _context()
    out = {"y": ctx.dropout(s["x"], c["p"], s["seed"], s["offset"], residual=s["residual"])}
    if c["train"]:
        out["dx"] = ctx.dropout(s["dy"], c["p"], s["seed"], s["offset"])
    return out


def run(state):
    op = state["case"]["op"]
    if own:
        return {"linear": _linear_own, "gated": _gated_own, "norm": _norm_own, "dropout": _dropout_own}[op](state)
    return {"linear": _linear_plain, "gated": _gated_plain, "norm": _norm_plain, "dropout": _dropout_plain}[op](state)


# ---------------------------------------------------------------------------------------------------- float64
def _act64(z, act):
    fn = torch.nn.functional
    return {"none": lambda: z, "relu": lambda: fn.relu(z), "gelu": lambda: fn.gelu(z), "silu": lambda: fn.silu(z),
            "gelu_tanh": lambda: fn.gelu(z, approximate="tanh"), "sigmoid": lambda: torch.sigmoid(z),
            "htanh": lambda: z.clamp(-1.0, 1.0)}[act]()


def _norm64(v, w, c, kind):
    mean = v.mean(1, keepdim=True) if kind == "layer" else 0.0
    y = (v - mean) / ((v - mean).pow(2).mean(1, keepdim=True) + EPS).sqrt() * w
    return y if c is None else y + c


def _kept64(shape, p, seed, offset):
    """The same published generator in unsigned 64-bit numpy arithmetic."""
    n = shape[0] * shape[1]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    at = np.arange((n + 3) // 4, dtype=np.uint64)
    word = [at & low, at >> half, np.full_like(at, offset & 0xFFFFFFFF), np.full_like(at, offset >> 32)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * word[0], np.uint64(0xCD9E8D57) * word[2]
        word = [(p1 >> half) ^ word[1] ^ np.uint64(key[0]), p1 & low, (p0 >> half) ^ word[3] ^ np.uint64(key[1]), p0 & low]
        key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
    return np.stack(word, 1).reshape(-1)[:n].reshape(shape) >= np.uint64(round(p * 2 ** 32))


def exact(case, seed):
    s = prepare(case, seed)
    train = case["train"]

    def leaf(name):
        t = s.get(name)
        return None if t is None else t.double().requires_grad_(train)

    if case["op"] == "linear":
        x, w, b = leaf("x"), leaf("W"), leaf("bias")
        out = _act64(x @ w.T if b is None else torch.addmm(b, x, w.T), case["act"])
        outs = {"y": out if s["residual"] is None else out + s["residual"].double()}
        wanted, seeds = {"dx": x, "dW": w, "db": b}, [s["dy"]]
    elif case["op"] == "gated":
        x, wg, wu = leaf("x"), leaf("Wg"), leaf("Wu")
        outs = {"h": _act64(x @ wg.T, case["act"]) * (x @ wu.T)}
        wanted, seeds = {"dx": x, "dWg": wg, "dWu": wu}, [s["dy"]]
    elif case["op"] == "norm":
        names = {"dx": "x", "dblock": "block", "dgate": "gate", "dpre_w": "pre_w", "dpre_c": "pre_c", "dpost_w": "post_w", "dpost_c": "post_c"}
        wanted = {k: leaf(v) for k, v in names.items()}
        p = wanted["dblock"]
        if case["post"]:
            p = _norm64(p, wanted["dpost_w"], wanted["dpost_c"], case["kind"])
        if case["gates"]:
            p = p * wanted["dgate"].repeat_interleave(s["per_gate"], 0)[: case["rows"]]
        stream = case["alpha"] * wanted["dx"] + p
        outs = {"stream": stream, "normed": _norm64(stream, wanted["dpre_w"], wanted["dpre_c"], case["kind"])}
        seeds = [s["dstream"], s["dnormed"]]
    else:
        kept = torch.from_numpy(_kept64(s["x"].shape, case["p"], s["seed"], s["offset"])).cuda()
        share = kept.double() / (1 - case["p"])
        outs = {"y": s["x"].double() * share + (0.0 if s["residual"] is None else s["residual"].double())}
        if train:
            outs["dx"] = s["dy"].double() * share
        return outs
    if train:
        wanted = {k: v for k, v in wanted.items() if v is not None}
        grads = torch.autograd.grad(list(outs.values()), list(wanted.values()), [g.double() for g in seeds])
        outs = {k: v.detach() for k, v in outs.items()} | dict(zip(wanted, grads))
    return outs
