"""Plain 64-bit forms of the real-valued operators, each with a bound on how far a correctly rounded float32 evaluation may be off.

Error model.  u is half a unit of the result's type (8, 11 and 24 significant bits: bfloat16 2^-8, float16 2^-11, float32 2^-24).  A float32 sum of K products is off by at
most (K + 32) 2^-23 times the sum of their magnitudes, whatever the order and also where additions truncate.  Fast exp and
division leave an activation within 2^-18 (|z| + 1); activations have slopes and curvatures below 1.2.  A value that is
rounded to 16 bits before a product (dz, dg, du) carries u of its own magnitude into it.
"""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
TINY = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -24, torch.float32: 1e-37}
ACT_ERR = 2.0 ** -18
KINKS = {"relu": (0.0,), "htanh": (-1.0, 1.0)}


def act(z, name):
    f = torch.nn.functional
    return {"none": lambda: z, "relu": lambda: f.relu(z), "gelu": lambda: f.gelu(z), "gelu_tanh": lambda: f.gelu(z, approximate="tanh"),
            "silu": lambda: f.silu(z), "sigmoid": lambda: torch.sigmoid(z), "htanh": lambda: z.clamp(-1, 1)}[name]()


def slope(z, name):
    z = z.detach().requires_grad_(True)
    return torch.autograd.grad(act(z, name).sum(), z)[0]


def gamma(k):
    return (k + 32) * 2.0 ** -23


def act_bound(z, ez, name):
    return 1.2 * ez + (0 if name == "none" else ACT_ERR * (z.abs() + 1))


def slope_bound(z, ez, name):
    """Error of act'(z) for z off by ez: all of it where a kink is that near."""
    e = 1.2 * ez + (0 if name == "none" else ACT_ERR * (z.abs() + 1))
    if name == "none":
        return torch.zeros_like(z)
    for k in KINKS.get(name, ()):
        e = torch.where((z - k).abs() <= ez, torch.ones_like(e), e)
    return e


def rounded(value, err, dtype):
    return err + UNIT[dtype] * (value.abs() + err) + TINY[dtype]


def linear(x, W, bias, residual, name, dy=None, keep_dz=False):
    """{output: (value, bound)} of the dense layer and, with dy, of its gradients."""
    dt = x.dtype
    x, W = x.double(), W.double()
    b = torch.zeros(W.shape[0], dtype=torch.float64, device=x.device) if bias is None else bias.double()
    z = x @ W.T + b
    ez = gamma(x.shape[1]) * (x.abs() @ W.abs().T + b.abs())
    y, ey = act(z, name), act_bound(z, ez, name)
    if residual is not None:
        y = residual.double() + y
        ey = ey + 2.0 ** -23 * (residual.double().abs() + y.abs())
    out = {"y": (y, rounded(y, ey, dt)), "pre": (z, ez + 1e-30)}
    if dy is None:
        return out
    d = dy.double()
    dz = d * slope(z, name)
    ed = d.abs() * slope_bound(z, ez, name)
    if name != "none":
        ed = rounded(dz, ed, dt)
    for key, a, ea, c, n in (("dx", dz, ed, W, W.shape[0]), ("dW", dz.T, ed.T, x, x.shape[0])):
        v = a @ c
        out[key] = (v, rounded(v, ea @ c.abs() + gamma(n) * ((a.abs() + ea) @ c.abs()), dt))
    v = dz.sum(0)
    out["db"] = (v, rounded(v, ed.sum(0) + gamma(x.shape[0]) * (dz.abs() + ed).sum(0), dt))
    return out


def gated(x, Wg, Wu, name, dh=None):
    dt = x.dtype
    x, Wg, Wu = x.double(), Wg.double(), Wu.double()
    g, u = x @ Wg.T, x @ Wu.T
    k = gamma(x.shape[1])
    eg, eu = k * (x.abs() @ Wg.abs().T), k * (x.abs() @ Wu.abs().T)
    a, ea = act(g, name), act_bound(g, eg, name)
    h = a * u
    out = {"h": (h, rounded(h, ea * (u.abs() + eu) + (a.abs() + ea) * eu + 2.0 ** -22 * h.abs(), dt)), "g": (g, eg + 1e-30), "u": (u, eu + 1e-30)}
    if dh is None:
        return out
    d = dh.double()
    s, es = slope(g, name), slope_bound(g, eg, name)
    dg, du = d * u * s, d * a
    edg = rounded(dg, d.abs() * (es * (u.abs() + eu) + (s.abs() + es) * eu) + 2.0 ** -22 * dg.abs(), dt)
    edu = rounded(du, d.abs() * ea + 2.0 ** -22 * du.abs(), dt)
    dx = dg @ Wg + du @ Wu
    sums = (dg.abs() + edg) @ Wg.abs() + (du.abs() + edu) @ Wu.abs()
    out["dx"] = (dx, rounded(dx, edg @ Wg.abs() + edu @ Wu.abs() + gamma(2 * Wg.shape[0]) * sums, dt))
    for key, t, e in (("dWg", dg, edg), ("dWu", du, edu)):
        v = t.T @ x
        out[key] = (v, rounded(v, e.T @ x.abs() + gamma(x.shape[0]) * ((t.abs() + e).T @ x.abs()), dt))
    return out


# Rows of D values: a thread adds at most 32 of them, then trees of depth 10: sums are off by at most 64 2^-24 of their magnitude.  A
# chain of mean, variance, root and products stays below ETA times the magnitude form, in which every difference is a sum.
ETA = 2.0 ** -17


def _norm(v, kind, eps):
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    r = 1 / ((v - mean).pow(2).mean(1, keepdim=True) + eps).sqrt()
    return (v - mean) * r, r


def _magnitude(v, kind, r):
    """Of the unit rows: |v| r + mean |v| r, and the relative error of r itself grows with the spread of |v| around the mean."""
    m = v.abs().mean(1, keepdim=True) if kind == "layer" else 0.0
    big = (v.abs() + m) * r
    return big + big * (big * big).mean(1, keepdim=True) if kind == "layer" else big * 2


def block_norm(x, block, n, ds=None, dn=None):
    """n: dict with kind, eps, alpha, post, pre, post_weight, post_shift, pre_weight, pre_shift, gate, rows_per_gate."""
    dt, M, D = x.dtype, x.shape[0], x.shape[1]
    f = lambda k, default: default if n.get(k) is None else n[k].double()  # noqa: E731
    kind, eps, alpha = n["kind"], n["eps"], n["alpha"]
    x = x.double()
    rows = torch.arange(M, device=x.device)
    gate = 1.0 if n.get("gate") is None else n["gate"].double()[rows // n["rows_per_gate"]]
    gabs = abs(gate) if isinstance(gate, float) else gate.abs()
    out = {}
    s, es, p, ep = alpha * x, 2.0 ** -23 * (alpha * x).abs(), None, None
    if block is not None:
        b = block.double()
        p, ep = b, torch.zeros_like(b)
        if n["post"]:
            bh, rb = _norm(b, kind, eps)
            ebh = ETA * _magnitude(b, kind, rb)
            w, c = f("post_weight", 1.0), f("post_shift", 0.0)
            p = bh * w + c
            ep = ebh * (abs(w) if isinstance(w, float) else w.abs()) + 2.0 ** -22 * p.abs()
        s = s + gate * p
        es = es + gabs * ep + 2.0 ** -22 * (s.abs() + gabs * p.abs())
    out["stream"] = (s, rounded(s, es, dt))
    if n["pre"]:
        sh, rs = _norm(s, kind, eps)
        # an error of s moves the unit row by r es, and its statistics by as much of the magnitudes
        esh = ETA * _magnitude(s, kind, rs) + 4 * rs * (es + es.mean(1, keepdim=True)) * (1 + sh.abs())
        w, c = f("pre_weight", torch.ones(D, dtype=torch.float64, device=x.device)), f("pre_shift", 0.0)
        v = sh * w + c
        out["normed"] = (v, rounded(v, esh * w.abs() + 2.0 ** -22 * v.abs(), dt))
    if ds is None and dn is None:
        return out
    col = gamma(M)
    T, eT = torch.zeros_like(s), torch.zeros_like(s)

    def back(e, ee, unit, eunit, r):
        m1, m2 = (e * unit).mean(1, keepdim=True), e.mean(1, keepdim=True) if kind == "layer" else 0.0
        v = r * (e - unit * m1 - m2)
        A, U = e.abs() + ee, unit.abs() + eunit
        am1 = (A * U).mean(1, keepdim=True)
        am2 = A.mean(1, keepdim=True) if kind == "layer" else 0.0
        err = r * (ee + eunit * am1 + U * ((ee * U).mean(1, keepdim=True) + (A * eunit).mean(1, keepdim=True)) +
                   (ee.mean(1, keepdim=True) if kind == "layer" else 0.0))
        rel = ETA + (eunit * U).mean(1, keepdim=True)          # of r
        return v, err + rel * r * (A + U * am1 + am2)

    if ds is not None:
        T = T + ds.double()
    if dn is not None and n["pre"]:
        d = dn.double()
        g, eg = back(d * w, 2.0 ** -23 * (d * w).abs(), sh, esh, rs)
        T, eT = T + g, eT + eg + 2.0 ** -23 * (T.abs() + g.abs())
        for key, t, e in (("dpre_weight", d * sh, d.abs() * esh), ("dpre_shift", d, 0 * d)):
            v = t.sum(0)
            out[key] = (v, rounded(v, e.sum(0) + col * (t.abs() + e).sum(0), dt))
    out["dx"] = (alpha * T, rounded(alpha * T, abs(alpha) * eT + 2.0 ** -23 * (alpha * T).abs(), dt))
    if block is None:
        return out
    dp, edp = gate * T, gabs * eT + 2.0 ** -23 * gabs * T.abs()
    if n.get("gate") is not None:
        G = n["gate"].shape[0]
        t, e = T * p, eT * (p.abs() + ep) + T.abs() * ep
        z = torch.zeros(G, D, dtype=torch.float64, device=x.device)
        v = z.index_add(0, rows // n["rows_per_gate"], t)
        out["dgate"] = (v, rounded(v, z.index_add(0, rows // n["rows_per_gate"], e + col * (t.abs() + e)), dt))
    if n["post"]:
        wv = f("post_weight", torch.ones(D, dtype=torch.float64, device=x.device))
        for key, t, e in (("dpost_weight", dp * bh, edp * (bh.abs() + ebh) + dp.abs() * ebh), ("dpost_shift", dp, edp)):
            v = t.sum(0)
            out[key] = (v, rounded(v, e.sum(0) + col * (t.abs() + e).sum(0), dt))
        dp, edp = back(dp * wv, edp * wv.abs() + 2.0 ** -23 * (dp * wv).abs(), bh, ebh, rb)
    out["dblock"] = (dp, rounded(dp, edp, dt))
    return out


def kept(rows, cols, p, seed, offset):
    """Philox4x32-10 in Python integers, one counter at a time: truth values [rows, cols]."""
    n, out = rows * cols, []
    for g in range((n + 3) // 4):
        c = [g & 0xFFFFFFFF, g >> 32, offset & 0xFFFFFFFF, offset >> 32]
        k = [seed & 0xFFFFFFFF, seed >> 32]
        for _ in range(10):
            a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
            c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
            k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
        out += [w >= round(p * 2 ** 32) for w in c]
    return torch.tensor(out[:n]).reshape(rows, cols)


def check(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape, f"{what}: shape {list(got.shape)}, expected {list(want.shape)}"
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} values outside their bound; worst at {int((off / bound).nan_to_num(math.inf).argmax())}: "
                           f"{float(off.max()):.3g} off, largest {float((off / bound).nan_to_num(math.inf).max()):.2f} times the bound")
