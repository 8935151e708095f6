"""Dense layer, gated projections, block norms and dropout on the GPU against their 64-bit forms: element types, ragged sizes,
pitches and bases off the 16-byte rule, empty and single dimensions, all gradients (also against differences), refusals,
other streams, offsets beyond 32 bits."""
import pytest
import torch

import real_reference as ref
from paper_1602_02830_b200 import binding, build

pytestmark = pytest.mark.gpu
BF, HF, FF = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def ctx():
    build.build()
    c = binding.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


def lend(ctx, n):
    ws = torch.full((max(n, 256) + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    ctx.set_workspace(ws[:max(n, 256)])
    return ws


def intact(ws, n):
    assert (ws[max(n, 256):] == 0x7F).all(), "written beyond the workspace"


class Maker:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def __call__(self, *shape, dtype=BF, scale=1.0, shift=0.0, pad=0, lead=0):
        """Normal values; pad: columns between rows, lead: elements before the first (moves the base off its alignment)."""
        t = torch.empty(*shape, device="cuda").normal_(shift, scale, generator=self.g).to(dtype)
        if not pad and not lead:
            return t
        rows, cols = shape if len(shape) == 2 else (1, shape[0])
        buf = torch.full((lead + rows * (cols + pad) + 8,), float("nan"), dtype=dtype, device="cuda")
        v = buf[lead:lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        v.copy_(t.view(rows, cols))
        return v if len(shape) == 2 else v[0]


class Framed:
    """An output inside a buffer of a sentinel, to see what is written around it."""

    def __init__(self, rows, cols, dtype, pad=0, lead=0):
        self.buf = torch.full((lead + rows * (cols + pad) + 64,), 77.0, dtype=dtype, device="cuda")
        self.t = self.buf[lead:lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]

    def check(self):
        seen = self.t.clone()
        self.t.fill_(77.0)
        assert (self.buf == 77.0).all(), "written outside the output"
        self.t.copy_(seen)


LINEAR = [  # M, N, K, type, act, bias, residual, pad, lead
    (1, 1, 1, BF, "none", True, True, 0, 0), (1, 4096, 512, BF, "none", True, True, 0, 0), (1, 10, 784, HF, "silu", False, False, 0, 0),
    (3, 257, 65, HF, "relu", True, False, 1, 1), (17, 1000, 1016, BF, "gelu", True, True, 8, 0), (64, 128, 4100, HF, "gelu_tanh", False, True, 0, 0),
    (65, 136, 72, BF, "htanh", True, True, 3, 2), (128, 256, 64, BF, "sigmoid", True, False, 0, 8), (200, 520, 264, HF, "none", False, True, 0, 0),
    (257, 511, 129, BF, "gelu", True, True, 5, 3), (300, 300, 2048, BF, "silu", True, False, 0, 0), (1030, 770, 392, HF, "relu", False, False, 0, 0),
    (513, 1024, 1023, BF, "none", True, True, 1, 0), (48, 2050, 2048, HF, "gelu_tanh", True, False, 0, 0), (2, 70000, 64, BF, "none", False, False, 0, 0),
    (16, 33, 9000, BF, "none", True, False, 0, 0), (1500, 24, 96, BF, "silu", True, True, 0, 0), (96, 640, 640, HF, "none", True, True, 0, 0),
]


@pytest.mark.parametrize("M,N,K,dtype,act,bias,residual,pad,lead", LINEAR)
def test_linear_forward(ctx, M, N, K, dtype, act, bias, residual, pad, lead):
    mk = Maker(M * 7 + N * 3 + K)
    x, W = mk(M, K, dtype=dtype, pad=pad, lead=lead), mk(N, K, dtype=dtype, scale=K ** -0.5, pad=pad, lead=lead)
    b = mk(N, dtype=dtype, lead=lead) if bias else None
    r = mk(M, N, dtype=dtype, pad=pad, lead=lead) if residual else None
    layer = ctx.make_linear(W, b, act)
    n = ctx.linear_workspace_bytes(layer, x)
    ws = lend(ctx, n)
    want = ref.linear(x, W, b, r, act)
    for lead_out in (0, 1):
        y, pre = Framed(M, N, dtype, pad, lead_out), Framed(M, N, FF, pad, lead_out)
        ctx.linear(layer, x, r, out=y.t, pre=pre.t)
        ctx.device_status()
        ref.check(y.t, *want["y"], "y")
        ref.check(pre.t, *want["pre"], "pre")
        y.check(), pre.check()
    ref.check(ctx.linear(layer, x, r), *want["y"], "y without pre")
    if r is not None:                                    # onto the residual itself
        ref.check(ctx.linear(layer, x, r, out=r), *want["y"], "y in place")
    intact(ws, n)


@pytest.mark.parametrize("M,N,K,dtype,act,bias,residual,pad,lead", LINEAR)
@pytest.mark.parametrize("kept", (True, False), ids=("kept", "again"))
def test_linear_backward(ctx, M, N, K, dtype, act, bias, residual, pad, lead, kept):
    if N * M * K > 1.5e9:
        pytest.skip("covered by smaller shapes")
    mk = Maker(M * 5 + N * 3 + K + 1)
    x, W = mk(M, K, dtype=dtype, pad=pad, lead=lead), mk(N, K, dtype=dtype, scale=K ** -0.5, pad=pad, lead=lead)
    b, dy = mk(N, dtype=dtype) if bias else None, mk(M, N, dtype=dtype, pad=pad, lead=lead)
    layer = ctx.make_linear(W, b, act)
    n = ctx.linear_workspace_bytes(layer, x, backward=True, dy=dy)
    ws = lend(ctx, n)
    pre = ctx.empty(M, N, dtype=FF) if kept else None
    if kept:
        ctx.linear(layer, x, pre=pre)
    want = ref.linear(x, W, b, None, act, dy)
    dx, dW, db = ctx.linear_backward(layer, dy, x, pre)
    ctx.device_status()
    ref.check(dx, *want["dx"], "dx")
    ref.check(dW, *want["dW"], "dW")
    if bias:
        ref.check(db, *want["db"], "db")
    assert (db is None) == (not bias)
    again = ctx.linear_backward(layer, dy, x, pre)
    for p, q in zip((dx, dW, db), again):
        assert p is None or torch.equal(p, q), "the same call gives other bits"
    only = ctx.linear_backward(layer, dy, x, pre, want_dx=False, want_db=False)
    assert only[0] is None and only[2] is None and torch.equal(only[1], dW)
    intact(ws, n)


def differences(loss, point, direction, h=1e-4):
    return float((loss(point + h * direction) - loss(point - h * direction)) / (2 * h))


def against_differences(grad, bound, loss, point, seed):
    v = torch.empty_like(point).normal_(generator=torch.Generator(device="cuda").manual_seed(seed))
    got, want = float((grad.double() * v).sum()), differences(loss, point, v)
    # the gradient's own bound along v, and the difference quotient's h^2 term and cancellation
    slack = float((bound * v.abs()).sum()) + 1e-6 * float(v.norm()) * (1 + abs(want))
    assert abs(got - want) <= slack, f"gradient along a direction {got}, difference quotient {want}, allowed {slack}"


@pytest.mark.parametrize("act", [a for a in binding.ACTIVATIONS if a not in ref.KINKS])
def test_linear_gradients_against_differences(ctx, act):
    mk = Maker(5)
    M, N, K = 33, 40, 24
    x, W, b, dy = mk(M, K, dtype=HF), mk(N, K, dtype=HF, scale=0.2), mk(N, dtype=HF), mk(M, N, dtype=HF)
    layer = ctx.make_linear(W, b, act)
    lend(ctx, ctx.linear_workspace_bytes(layer, x, backward=True))
    pre = ctx.empty(M, N, dtype=FF)
    ctx.linear(layer, x, pre=pre)
    grads = dict(zip(("dx", "dW", "db"), ctx.linear_backward(layer, dy, x, pre)))
    want = ref.linear(x, W, b, None, act, dy)
    f = lambda p, q, r: (ref.act(p @ q.T + r, act) * dy.double()).sum()  # noqa: E731
    X, Y, Z = x.double(), W.double(), b.double()
    against_differences(grads["dx"], want["dx"][1], lambda t: f(t, Y, Z), X, 1)
    against_differences(grads["dW"], want["dW"][1], lambda t: f(X, t, Z), Y, 2)
    against_differences(grads["db"], want["db"][1], lambda t: f(X, Y, t), Z, 3)


GATED = [  # M, N, K, type, act, pad, lead
    (1, 1, 1, BF, "silu", 0, 0), (1, 8192, 256, BF, "silu", 0, 0), (1, 513, 100, HF, "gelu", 1, 1), (5, 96, 2048, HF, "gelu_tanh", 0, 0),
    (16, 700, 264, BF, "sigmoid", 0, 8), (48, 1375, 512, HF, "gelu_tanh", 0, 0), (65, 129, 130, BF, "relu", 3, 1), (130, 264, 1000, BF, "silu", 8, 0),
    (256, 512, 256, HF, "htanh", 0, 0), (333, 515, 72, BF, "none", 0, 0), (700, 384, 1024, BF, "silu", 0, 0), (1025, 640, 136, HF, "gelu", 0, 0),
    (7, 33, 9000, BF, "silu", 0, 0),
]


@pytest.mark.parametrize("M,N,K,dtype,act,pad,lead", GATED)
def test_gated(ctx, M, N, K, dtype, act, pad, lead):
    mk = Maker(M + N * 3 + K)
    x = mk(M, K, dtype=dtype, pad=pad, lead=lead)
    Wg, Wu = mk(N, K, dtype=dtype, scale=K ** -0.5, pad=pad, lead=lead), mk(N, K, dtype=dtype, scale=K ** -0.5, pad=2 * pad)
    dh = mk(M, N, dtype=dtype, pad=pad, lead=lead)
    layer = ctx.make_gated(Wg, Wu, act)
    n = ctx.gated_workspace_bytes(layer, x, backward=True)
    ws = lend(ctx, n)
    want = ref.gated(x, Wg, Wu, act, dh)
    pre = ctx.empty(2, M, N, dtype=FF)
    for lead_out in (0, 1):
        h = Framed(M, N, dtype, pad, lead_out)
        ctx.gated(layer, x, out=h.t, pre=pre if lead_out else None)
        ctx.device_status()
        ref.check(h.t, *want["h"], "h")
        h.check()
    ref.check(pre[0], *want["g"], "g")
    ref.check(pre[1], *want["u"], "u")
    for kept in (pre, None):
        got = ctx.gated_backward(layer, dh, x, kept)
        ctx.device_status()
        for key, t in zip(("dx", "dWg", "dWu"), got):
            ref.check(t, *want[key], key)
        assert all(torch.equal(p, q) for p, q in zip(got, ctx.gated_backward(layer, dh, x, kept))), "the same call gives other bits"
        only = ctx.gated_backward(layer, dh, x, kept, want_dW=False)
        assert torch.equal(only[0], got[0]) and only[1] is None and only[2] is None
    intact(ws, n)


@pytest.mark.parametrize("act", [a for a in binding.ACTIVATIONS if a not in ref.KINKS])
def test_gated_gradients_against_differences(ctx, act):
    mk = Maker(6)
    M, N, K = 20, 48, 32
    x, Wg, Wu, dh = mk(M, K, dtype=HF), mk(N, K, dtype=HF, scale=0.2), mk(N, K, dtype=HF, scale=0.2), mk(M, N, dtype=HF)
    layer = ctx.make_gated(Wg, Wu, act)
    lend(ctx, ctx.gated_workspace_bytes(layer, x, backward=True))
    dx, dWg, dWu = ctx.gated_backward(layer, dh, x)
    want = ref.gated(x, Wg, Wu, act, dh)
    f = lambda p, q, r: (ref.act(p @ q.T, act) * (p @ r.T) * dh.double()).sum()  # noqa: E731
    X, G, U = x.double(), Wg.double(), Wu.double()
    against_differences(dx, want["dx"][1], lambda t: f(t, G, U), X, 1)
    against_differences(dWg, want["dWg"][1], lambda t: f(X, t, U), G, 2)
    against_differences(dWu, want["dWu"][1], lambda t: f(X, G, t), U, 3)


@pytest.mark.parametrize("M,N,K", [(0, 8, 8), (4, 0, 8), (4, 8, 0), (0, 8, 0), (4, 0, 0)])
def test_empty_products(ctx, M, N, K):
    mk = Maker(3)
    x, W, b, r = mk(M, K), mk(N, K), mk(N), mk(M, N)
    layer, glu = ctx.make_linear(W, b, "gelu"), ctx.make_gated(W, W.clone(), "silu")
    lend(ctx, max(ctx.linear_workspace_bytes(layer, x, backward=True), ctx.gated_workspace_bytes(glu, x, backward=True)))
    want = ref.linear(x, W, b, r, "gelu", r)
    pre = ctx.empty(M, N, dtype=FF)
    ref.check(ctx.linear(layer, x, r, pre=pre), *want["y"], "y")
    for kept in (pre, None):
        for key, t in zip(("dx", "dW", "db"), ctx.linear_backward(layer, r, x, kept)):
            ref.check(t, *want[key], key)
    assert (ctx.gated(glu, x) == 0).all()
    assert all((t == 0).all() for t in ctx.gated_backward(glu, r, x))
    ctx.device_status()


def test_non_finite_inputs_stay_in_their_rows(ctx):
    mk = Maker(4)
    for M in (5, 300):
        x, W = mk(M, 200), mk(130, 200, scale=0.1)
        clean = x.clone()
        x[2, 7], x[4, 0] = float("nan"), float("inf")
        for run in (lambda t: ctx.linear(ctx.make_linear(W, None, "relu"), t), lambda t: ctx.gated(ctx.make_gated(W, W), t)):
            y, z = run(x), run(clean)
            rows = torch.ones(M, dtype=torch.bool, device="cuda")
            rows[2] = rows[4] = False
            assert torch.equal(y[rows], z[rows]) and y[2].isnan().all() and not y[4].isfinite().all()
        s, n = ctx.block_norm(ctx.make_block_norm(200, BF), x)
        t, m = ctx.block_norm(ctx.make_block_norm(200, BF), clean)
        assert torch.equal(n[rows], m[rows]) and n[2].isnan().all()


NORM = [  # M, D, type, kind, post, pre, gate rows, alpha, weights, shifts, block, pad, lead
    (1, 1, FF, "rms", True, True, 1, 1.0, True, True, True, 0, 0), (1, 4096, BF, "rms", True, True, 1, 1.0, True, False, True, 0, 0),
    (3, 7, HF, "layer", True, True, 0, 0.5, True, True, True, 1, 1), (64, 256, BF, "rms", False, True, 0, 1.0, True, False, True, 0, 0),
    (100, 1011, FF, "layer", False, True, 8, 0.5, True, True, True, 0, 0), (257, 1024, HF, "layer", True, True, 3, 2.0, True, True, True, 8, 0),
    (50, 2050, BF, "rms", True, False, 50, 1.0, False, False, True, 0, 0), (400, 784, FF, "rms", True, True, 400, 1.0, True, False, True, 0, 4),
    (33, 8192, BF, "layer", True, True, 4, 1.0, True, True, True, 0, 0), (9, 8200, HF, "rms", True, True, 2, 1.0, True, True, True, 0, 0),
    (5, 16384, FF, "layer", True, True, 1, 1.0, True, True, True, 0, 0), (4, 32768, BF, "rms", True, True, 2, 0.7, True, True, True, 0, 0),
    (3, 32767, BF, "layer", True, True, 1, 1.0, True, True, True, 0, 1), (700, 128, BF, "rms", False, True, 0, 1.0, True, False, False, 0, 0),
    (20, 96, FF, "layer", False, True, 0, 1.0, False, False, False, 0, 0), (600, 520, BF, "rms", False, False, 1, 1.0, False, False, True, 0, 0),
    (1000, 64, HF, "rms", True, True, 7, 1.0, True, True, True, 3, 0),
]


@pytest.mark.parametrize("M,D,dtype,kind,post,pre,gates,alpha,weights,shifts,block,pad,lead", NORM)
def test_block_norm(ctx, M, D, dtype, kind, post, pre, gates, alpha, weights, shifts, block, pad, lead):
    mk = Maker(M + D)
    x, b = mk(M, D, dtype=dtype, scale=2.0, pad=pad, lead=lead), mk(M, D, dtype=dtype, shift=0.3, pad=pad) if block else None
    par = {"kind": kind, "eps": 1e-5, "alpha": alpha, "post": post, "pre": pre, "rows_per_gate": -(-M // gates) if gates else None,
           "gate": mk(gates, D, dtype=dtype, shift=0.5, pad=pad) if gates else None}
    for name, on in (("post", post), ("pre", pre)):
        par[name + "_weight"] = mk(D, dtype=dtype, scale=0.2, shift=1.0, lead=lead) if on and weights else None
        par[name + "_shift"] = mk(D, dtype=dtype, scale=0.2) if on and shifts else None
    ds, dn = mk(M, D, dtype=dtype, pad=pad, lead=lead), mk(M, D, dtype=dtype) if pre else None
    layer = ctx.make_block_norm(D, dtype, **par)
    want = ref.block_norm(x, b, par, ds, dn)
    n = ctx.block_norm_workspace_bytes(layer, M)
    ws = lend(ctx, n)
    stats = ctx.empty(M, 4, dtype=FF)
    stream, normed = Framed(M, D, dtype, pad, lead), Framed(M, D, dtype, pad, 0)
    ctx.block_norm(layer, x, b, stream=stream.t, normed=normed.t if pre else None, stats=stats)
    ref.check(stream.t, *want["stream"], "stream")
    if pre:
        ref.check(normed.t, *want["normed"], "normed")
    stream.check(), normed.check()
    got = ctx.block_norm_backward(layer, ds, dn, x, b, stats)
    for key, t in got.items():
        if t is not None:
            if key in want:
                ref.check(t, *want[key], key)
        else:
            assert key not in want or key.startswith(("dp", "dg"))
    again = ctx.block_norm_backward(layer, ds, dn, x, b, stats)
    assert all(t is None or torch.equal(t, again[k]) for k, t in got.items()), "the same call gives other bits"
    if pre:                                                # each of the incoming gradients alone
        for ds1, dn1 in ((ds, None), (None, dn)):
            part = ref.block_norm(x, b, par, ds1, dn1)
            for key, t in ctx.block_norm_backward(layer, ds1, dn1, x, b, stats).items():
                if t is not None:
                    ref.check(t, *part.get(key, (torch.zeros_like(t).double(), 0)), key)
    kept = x.clone()
    s2, _ = ctx.block_norm(layer, kept, b, stream=kept)      # onto the stream itself
    ref.check(s2, *want["stream"], "stream in place")
    intact(ws, n)


@pytest.mark.parametrize("kind,shifts", [("rms", False), ("layer", True)])
@pytest.mark.parametrize("dtype", (BF, FF))
@pytest.mark.parametrize("D", (8, 248, 256, 264, 504, 1000, 1952, 2048, 2056, 4088, 4096, 4104, 8192, 8200, 16384))
def test_block_norm_of_every_team(ctx, D, dtype, kind, shifts):
    """Widths around every change of team, slots and stages."""
    mk = Maker(D)
    M = 11
    x, b, ds, dn = mk(M, D, dtype=dtype, scale=2.0), mk(M, D, dtype=dtype), mk(M, D, dtype=dtype), mk(M, D, dtype=dtype)
    par = {"kind": kind, "eps": 1e-5, "alpha": 1.0, "post": True, "pre": True, "rows_per_gate": 6, "gate": mk(2, D, dtype=dtype, shift=0.5)}
    par |= {k: mk(D, dtype=dtype, scale=0.2, shift=1.0) for k in ("post_weight", "pre_weight")}
    par |= {k: mk(D, dtype=dtype, scale=0.2) if shifts else None for k in ("post_shift", "pre_shift")}
    layer = ctx.make_block_norm(D, dtype, **par)
    n = ctx.block_norm_workspace_bytes(layer, M)
    ws = lend(ctx, n)
    stats = ctx.empty(M, 4, dtype=FF)
    want = ref.block_norm(x, b, par, ds, dn)
    for key, t in zip(("stream", "normed"), ctx.block_norm(layer, x, b, stats=stats)):
        ref.check(t, *want[key], key)
    for key, t in ctx.block_norm_backward(layer, ds, dn, x, b, stats).items():
        if t is not None:
            ref.check(t, *want[key], key)
    intact(ws, n)


def test_block_norm_gradients_against_differences(ctx):
    mk = Maker(8)
    M, D = 12, 40
    for kind in binding.NORMS:
        x, b, ds, dn = (mk(M, D, dtype=FF) for _ in range(4))
        par = {"kind": kind, "eps": 1e-5, "alpha": 0.8, "post": True, "pre": True, "rows_per_gate": 5, "gate": mk(3, D, dtype=FF)}
        par |= {k: mk(D, dtype=FF, shift=1.0) for k in ("post_weight", "post_shift", "pre_weight", "pre_shift")}
        layer = ctx.make_block_norm(D, FF, **par)
        lend(ctx, ctx.block_norm_workspace_bytes(layer, M))
        stats = ctx.empty(M, 4, dtype=FF)
        ctx.block_norm(layer, x, b, stats=stats)
        got = ctx.block_norm_backward(layer, ds, dn, x, b, stats)
        want = ref.block_norm(x, b, par, ds, dn)

        for i, (key, name, at) in enumerate((("dx", "x", x), ("dblock", "block", b), ("dgate", "gate", par["gate"]),
                                             *(("d" + k, k, par[k]) for k in ("post_weight", "post_shift", "pre_weight", "pre_shift")))):
            # the 64-bit form takes 64-bit arguments; bounds are those of the float32 results
            big = {"x": x.double(), "block": b.double()} | {k: v.double() for k, v in par.items() if torch.is_tensor(v)}

            def along(t, name=name):
                return loss64({**big, name: t}, par, ds, dn)

            against_differences(got[key], want[key][1], along, at.double(), i)


def loss64(p, par, ds, dn):
    def norm(v, w, c):
        m = v.mean(1, keepdim=True) if par["kind"] == "layer" else 0.0
        return (v - m) / ((v - m).pow(2).mean(1, keepdim=True) + par["eps"]).sqrt() * w + c
    rows = torch.arange(p["x"].shape[0], device="cuda") // par["rows_per_gate"]
    s = par["alpha"] * p["x"] + p["gate"][rows] * norm(p["block"], p["post_weight"], p["post_shift"])
    return (s * ds.double()).sum() + (norm(s, p["pre_weight"], p["pre_shift"]) * dn.double()).sum()


def test_block_norm_of_no_rows(ctx):
    layer = ctx.make_block_norm(16, BF, kind="layer", post=True, post_weight=Maker(1)(16), pre_weight=Maker(2)(16), pre_shift=Maker(3)(16))
    x = ctx.empty(0, 16, dtype=BF)
    ctx.set_workspace(None)
    s, n = ctx.block_norm(layer, x, x)
    assert s.shape == n.shape == (0, 16)
    got = ctx.block_norm_backward(layer, x, x, x, x, ctx.empty(0, 4, dtype=FF))
    assert all((got[k] == 0).all() for k in ("dpost_weight", "dpre_weight", "dpre_shift"))


DROP = [(1, 1, FF, 0.5, True, 0, 0), (1, 4099, BF, 0.1, True, 0, 0), (7, 13, HF, 0.3, False, 0, 0), (33, 64, BF, 0.5, True, 8, 0),
        (33, 64, FF, 0.9, False, 3, 1), (5, 101, BF, 0.0, True, 2, 3), (6, 72, HF, 1.0, True, 0, 0), (128, 40, BF, 0.25, True, 0, 4)]


@pytest.mark.parametrize("M,D,dtype,p,residual,pad,lead", DROP)
def test_dropout(ctx, M, D, dtype, p, residual, pad, lead):
    mk = Maker(M + D)
    x, r = mk(M, D, dtype=dtype, shift=3.0, pad=pad, lead=lead), mk(M, D, dtype=dtype, pad=pad) if residual else None
    seed, offset = 0xFEDCBA9876543210, 0x123456789ABCDEF
    keep = ref.kept(M, D, p, seed, offset).cuda()
    scaled = x.double() / (1 - p) if p < 1 else torch.zeros_like(x).double()
    want = torch.where(keep, scaled, 0.0) + (r.double() if residual else 0.0)
    bound = ref.rounded(want, 2.0 ** -22 * (scaled.abs() + want.abs()), dtype)
    y = Framed(M, D, dtype, pad, lead)
    ctx.dropout(x, p, seed, offset, residual=r, out=y.t)
    ref.check(y.t, want, bound, "y")
    y.check()
    bad = x.clone()
    bad[~keep] = float("nan")                              # what is dropped is not looked at
    assert torch.equal(ctx.dropout(bad, p, seed, offset, residual=r), y.t)
    g = ctx.dropout(torch.ones_like(x), p, seed, offset)   # the backward pass of a gradient of ones
    assert torch.equal(g != 0, keep)
    assert torch.equal(ctx.dropout(bad, p, seed, offset, residual=r, out=bad), y.t), "in place"


def test_dropout_share_and_seeds(ctx):
    x = torch.ones(2000, 1000, dtype=FF, device="cuda")
    for p in (0.1, 0.5, 0.875):
        y = ctx.dropout(x, p, 11)
        n = x.numel()
        assert abs(float((y != 0).sum()) - n * (1 - p)) < 6 * (n * p * (1 - p)) ** 0.5          # six deviations of a binomial
        for other in (ctx.dropout(x, p, 12), ctx.dropout(x, p, 11, 1), ctx.dropout(x, p, 11 + (1 << 32)), ctx.dropout(x, p, 11, 1 << 32)):
            same = float(((other != 0) == (y != 0)).double().mean())
            assert abs(same - (p * p + (1 - p) ** 2)) < 0.01


def test_rows_far_apart(ctx):
    """Offsets beyond 32 bits: three rows in a buffer of 2.3 G elements."""
    ld = 1_150_000_008
    buf = torch.empty(2 * ld + 4096, dtype=HF, device="cuda")
    mk = Maker(9)
    x = buf.as_strided((3, 264), (ld, 1))
    x.copy_(mk(3, 264, dtype=HF))
    W, near = mk(40, 264, dtype=HF, scale=0.1), x.clone()
    layer, glu, norm = ctx.make_linear(W), ctx.make_gated(W, W), ctx.make_block_norm(264, HF)
    lend(ctx, 1 << 22)
    out = buf.as_strided((3, 264), (ld, 1), 2048)
    assert torch.equal(ctx.linear(layer, x), ctx.linear(layer, near))
    assert torch.equal(ctx.gated(glu, x), ctx.gated(glu, near))
    assert torch.equal(ctx.block_norm(norm, x, near, stream=out)[0], ctx.block_norm(norm, near, near)[0])
    assert torch.equal(ctx.dropout(x, 0.5, 3, out=out), ctx.dropout(near, 0.5, 3))
    dy = mk(3, 40, dtype=HF)
    assert torch.equal(ctx.linear_backward(layer, dy, x)[1], ctx.linear_backward(layer, dy, near)[1])
    ctx.device_status()


def test_another_stream():
    """Tensors of torch's current stream through a context of another one: results whole, memory kept until they are used."""
    side = torch.cuda.Stream()
    c = binding.Context(0, side)
    mk = Maker(12)
    W, x = mk(512, 512, scale=0.05), mk(300, 512)
    layer = c.make_linear(W, None, "gelu")
    want = ref.linear(x, W, None, None, "gelu")
    side.wait_stream(torch.cuda.current_stream())
    y = c.linear(layer, x)
    junk = [torch.full((300, 512), 9.0, dtype=BF, device="cuda") for _ in range(8)]       # would reuse y's memory if it were free
    torch.cuda.current_stream().wait_stream(side)
    ref.check(y, *want["y"], "y")
    del junk
    side.synchronize()
    c.close()


@pytest.mark.parametrize("M", (3, 700), ids=("few", "pairs"))
def test_waits_that_run_out(M):
    """With the producers switched off every wait of the products runs out: a status, no hang, and the context works afterwards."""
    c = binding.Context(0)
    mk = Maker(14)
    x, W = mk(M, 512), mk(1000, 512, scale=0.05)
    layer, glu, dy = c.make_linear(W), c.make_gated(W, W), mk(M, 1000)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    c.set_workspace(ws)
    c.set_wait_limit_ns(20_000_000)
    for call in (lambda: c.linear(layer, x), lambda: c.gated(glu, x), lambda: c.linear_backward(layer, dy, x)):
        c.debug_drop_loads(True)
        call()
        with pytest.raises(binding.BnnError) as e:
            c.device_status()
        assert e.value.status == -5
        c.debug_drop_loads(False)
        call()
        c.device_status()
    ref.check(c.linear(layer, x), *ref.linear(x, W, None, None, "none")["y"], "y after failures")
    c.close()


def test_captured_in_a_graph():
    """The calls of a training step replayed from a CUDA graph give the bits of the calls themselves."""
    side = torch.cuda.Stream()
    c = binding.Context(0, side)
    mk = Maker(15)
    x, W, Wg, dy = mk(130, 256), mk(256, 640, scale=0.05), mk(640, 256, scale=0.05), mk(130, 256)
    layer, glu, norm = c.make_linear(W), c.make_gated(Wg, Wg), c.make_block_norm(256, BF, post=True, pre_weight=mk(256, shift=1.0))
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    c.set_workspace(ws)

    def step():
        pre, stats = c.empty(2, 130, 640, dtype=FF), c.empty(130, 4, dtype=FF)
        h = c.gated(glu, x, pre=pre)
        b = c.dropout(c.linear(layer, h), 0.25, 5)
        s, n = c.block_norm(norm, x, b, stats=stats)
        back = c.block_norm_backward(norm, dy, dy, x, b, stats)
        dh, dW, _ = c.linear_backward(layer, back["dblock"], h)
        return [s, n, back["dx"], back["dpre_weight"], dW, *c.gated_backward(glu, dh, x, pre)]

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [t.clone() for t in step()]
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = step()
        for _ in range(3):
            for t in got:
                t.fill_(9.0)
            graph.replay()
    side.synchronize()
    c.device_status()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    c.close()


def test_refusals(ctx):
    mk = Maker(2)
    x, W, b = mk(4, 64), mk(32, 64), mk(32)
    layer = ctx.make_linear(W, b, "gelu")
    for bad in (lambda: ctx.make_linear(W.float()), lambda: ctx.make_linear(W, act="tanh"), lambda: ctx.make_linear(W, b[:5]),
                lambda: ctx.make_linear(W.t()), lambda: ctx.make_gated(W, W.half()), lambda: ctx.make_gated(W, W[:4]),
                lambda: ctx.linear(layer, x.half()), lambda: ctx.linear(layer, x[:, :8]), lambda: ctx.linear(layer, x.cpu()),
                lambda: ctx.linear(layer, x, residual=x), lambda: ctx.linear(layer, mk(64, 4).t()), lambda: ctx.linear(layer, x[:1].expand(4, 64)),
                lambda: ctx.linear(layer, x, pre=ctx.empty(4, 32, dtype=BF)), lambda: ctx.dropout(x, 1.5, 0), lambda: ctx.dropout(x, 0.5, -1),
                lambda: ctx.dropout(x.double(), 0.5, 0), lambda: ctx.make_block_norm(64, BF, kind="batch"),
                lambda: ctx.make_block_norm(64, BF, gate=mk(3, 64)), lambda: ctx.block_norm(ctx.make_block_norm(32, BF), x),
                lambda: ctx.block_norm(ctx.make_block_norm(64, BF, gate=mk(1, 64), rows_per_gate=2), x, x),
                lambda: ctx.gated(ctx.make_gated(W, W), x, pre=ctx.empty(4, 2, 32, dtype=FF))):
        with pytest.raises(ValueError):
            bad()
    def status(call):
        with pytest.raises(binding.BnnError) as e:
            call()
        return e.value.status

    ctx.set_workspace(None)
    assert status(lambda: ctx.linear_backward(layer, mk(4, 32), x)) == -3
    assert status(lambda: ctx.gated_backward(ctx.make_gated(W, W), mk(4, 32), x)) == -3
    norm = ctx.make_block_norm(64, BF, pre_weight=mk(64))
    assert status(lambda: ctx.block_norm_backward(norm, x, x, x, x, ctx.empty(4, 4, dtype=FF))) == -3
    assert status(lambda: ctx.block_norm_backward(norm, x, x, x, x)) == -1                 # no statistics
    assert status(lambda: ctx.block_norm(ctx.make_block_norm(64, BF, post=True), x)) == -1  # a norm after no block
    assert status(lambda: ctx.block_norm(ctx.make_block_norm(32769, BF), ctx.empty(1, 32769, dtype=BF))) == -1
