"""Microscaled operators on the GPU against their 64-bit forms: quantisation bit by bit, norms with a microscaled result, products of every pair of
formats on both kernels, microscaled results, gradients straight through the rounding, edges of masks, sizes, strides and streams."""
import threading

import pytest
import torch

import mx_reference as mx
import real_reference as ref
from paper_1602_02830_b200 import binding, build

pytestmark = pytest.mark.gpu
BF, HF, FF = torch.bfloat16, torch.float16, torch.float32
FORMATS = ("e4m3", "e2m1")
PAIRS = (("e4m3", "e4m3"), ("e4m3", "e2m1"), ("e2m1", "e2m1"))


@pytest.fixture(scope="module")
def ctx():
    build.build()
    c = binding.Context(0)
    yield c
    torch.cuda.synchronize()
    c.close()


class Maker:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def __call__(self, *shape, dtype=BF, scale=1.0, shift=0.0, pad=0, lead=0, spread=0.0):
        """Normal values; pad: columns between rows, lead: elements before the first; spread: of the columns' sizes (natural logarithm)."""
        t = torch.empty(*shape, device="cuda").normal_(shift, scale, generator=self.g)
        if spread:
            t = t * torch.empty(shape[-1], device="cuda").normal_(0.0, spread, generator=self.g).exp()
        t = t.to(dtype)
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


def framed_mx(ctx, rows, cols, fmt):
    """A microscaled matrix between sentinels; what is behind its last row has to stay."""
    L, code = binding.lib(), binding.MX_FORMATS[fmt]
    n, s = rows * L.bnn_mx_ld(code, cols), L.bnn_mx_scale_bytes(rows, cols)
    room, marks = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda"), torch.full((s + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    q = binding.MxMatrix(fmt, rows, cols, room[:n].view(rows, -1) if n else room[:0].view(rows, 0), marks[:s], 0)

    def intact():
        assert (room[n:] == 0xA5).all() and (marks[s:] == 0xA5).all(), "written behind the matrix"
        if rows and cols:
            r = torch.arange(-(-rows // 128) * 128)[:, None]
            at = ((r // 128) * -(-cols // 128) + torch.arange(-(-cols // 128))[None, :])[:, :, None] * 512 + (r % 32 * 16 + r % 128 // 32 * 4)[:, :, None] + torch.arange(4)
            assert (marks[:s].cpu()[at[rows:].reshape(-1)] == 0xA5).all(), "scales of rows that do not exist"
    return q, intact


def same(a, b):
    """Equal values, NaN with NaN."""
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(torch.nan_to_num(a, 0.0), torch.nan_to_num(b, 0.0))


# ---------------------------------------------------------------------------------------------------- quantisation
QUANTIZE = [  # M, K, pad, lead
    (1, 1, 0, 0), (1, 31, 0, 0), (1, 32, 0, 0), (2, 33, 0, 1), (5, 127, 1, 0), (3, 128, 0, 0), (33, 129, 7, 3), (128, 256, 0, 0), (129, 257, 0, 0), (7, 1011, 3, 2),
    (130, 1000, 8, 8), (1, 4096, 0, 0), (64, 520, 4, 4), (300, 2050, 0, 0), (17, 8192, 2, 0),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", (FF, BF, HF), ids=("f32", "bf16", "f16"))
@pytest.mark.parametrize("M,K,pad,lead", QUANTIZE)
def test_quantize_is_exact(ctx, M, K, pad, lead, dtype, fmt):
    x = Maker(M * 7 + K)(M, K, dtype=dtype, pad=pad, lead=lead, spread=2.0)
    want = mx.quantize(x.double(), fmt)
    q, intact = framed_mx(ctx, M, K, fmt)
    out = Framed(M, K, dtype, pad, lead)
    assert ctx.mx_quantize(x, out=q, values=out.t) is q
    intact(), out.check()
    values, padding, scales = mx.read(q)
    assert torch.equal(values, want.cpu()), "the bytes do not stand for the nearest elements"
    assert (padding == 0).all(), "padding that is not zero"
    assert torch.equal(out.t, want.to(dtype)), "represented values"
    for t in (FF, BF, HF):
        back = Framed(M, K, t, pad, lead)
        ctx.mx_values(q, t, out=back.t)
        assert torch.equal(back.t, want.to(t)), "values read back"
        back.check()
    again, _ = framed_mx(ctx, M, K, fmt)
    ctx.mx_quantize(want.float(), out=again)
    assert torch.equal(mx.read(again)[0], values) and torch.equal(mx.read(again)[2], scales), "represented values, quantised again, change"
    ctx.mx_quantize(x, out=q, values=x)                  # onto the source itself
    assert torch.equal(x, want.to(dtype))


@pytest.mark.parametrize("fmt", FORMATS)
def test_quantize_borders_and_extremes(ctx, fmt):
    """Every element, every border of two and its neighbours on either side, at scales from the smallest to the largest; all zero, subnormal and saturating blocks."""
    t = mx.table(fmt).float()
    mid = (t[1:] + t[:-1]) / 2
    v = torch.cat([t, mid, torch.nextafter(mid, t[1:]), torch.nextafter(mid, t[:-1]), t[-1:] * 1.1, t[-1:] * 1.1428])
    rows = []
    for e in (-126 + 0, -100, -3, 0, 7, 60, 119 if fmt == "e4m3" else 125):
        b = torch.nn.functional.pad(v, (0, -len(v) % 31)).view(-1, 31)
        b = torch.cat([t[-1:].expand(len(b), 1), b], 1)              # each block has the largest element, which sets its exponent
        rows.append(torch.ldexp(b, torch.tensor(float(e))).reshape(-1))
    x = torch.stack(rows)
    x = torch.cat([x, -x, torch.zeros_like(x[:1]), torch.full_like(x[:1], 1e-45), torch.full_like(x[:1], 3e-39), torch.full_like(x[:1], 3.4e38)]).cuda()
    q = ctx.mx_quantize(x, fmt)
    want = mx.quantize(x.double(), fmt).cpu()
    assert torch.equal(mx.read(q)[0], want)
    assert torch.equal(ctx.mx_values(q).double().cpu(), want)        # 2^-127 itself is a subnormal of float32


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("K", (96, 97))
def test_quantize_not_finite(ctx, K, fmt):
    x = Maker(K)(6, K, dtype=FF)
    x[1, 5], x[2, 40], x[3, 95], x[4, 0] = float("nan"), float("inf"), -float("inf"), torch.finfo(FF).max
    out = torch.empty_like(x)
    q = ctx.mx_quantize(x, fmt, values=out)
    want = mx.quantize(x.double(), fmt)
    assert same(out.double(), want) and same(ctx.mx_values(q).double(), want)
    assert want.isnan().sum() == 96 and (mx.read(q)[2] == 255).sum() == 3
    # a block that is NaN makes the outputs that it enters NaN and no others: as a row of x, and as a row of the weights
    clean = ctx.mx_quantize(torch.nan_to_num(x, 0.0, 0.0, 0.0), fmt)
    y = ctx.mx_linear(ctx.make_mx_linear(clean), q)
    assert y.isnan().all(1).tolist() == [False, True, True, True, False, False] and y[[0, 5]][:, [0, 1, 2, 3, 5]].isfinite().all()      # (row 4 is near the largest float)
    y = ctx.mx_linear(ctx.make_mx_linear(q), clean)
    assert y.isnan().all(0).tolist() == [False, True, True, True, False, False] and y[[0, 1, 2, 3, 5]][:, [0, 5]].isfinite().all()


def test_empty_matrices(ctx):
    for rows, cols in ((0, 64), (4, 0), (0, 0)):
        q = ctx.mx_quantize(torch.empty(rows, cols, dtype=BF, device="cuda"), "e4m3")
        assert ctx.mx_values(q, BF).shape == (rows, cols)
    W, b = ctx.mx_quantize(torch.randn(40, 0, device="cuda").to(BF)), torch.randn(40, device="cuda").to(BF)
    pre = torch.full((3, 40), 5.0, device="cuda")
    y = ctx.mx_linear(ctx.make_mx_linear(W, b, "relu"), ctx.make_mx(3, 0), pre=pre)             # the empty sum: the bias alone
    assert torch.equal(y, b.relu().expand(3, 40)) and torch.equal(pre, b.float().expand(3, 40))
    assert (ctx.mx_gated(ctx.make_mx_gated(W, W), ctx.make_mx(3, 0)) == 0).all()
    h = ctx.mx_gated(ctx.make_mx_gated(W, W), ctx.make_mx(3, 0), out=ctx.make_mx(3, 40))
    assert (ctx.mx_values(h) == 0).all()
    W = ctx.mx_quantize(torch.randn(40, 64, device="cuda").to(BF))
    assert ctx.mx_linear(ctx.make_mx_linear(W), ctx.make_mx(0, 64)).shape == (0, 40)
    assert ctx.mx_linear(ctx.make_mx_linear(ctx.make_mx(0, 64)), ctx.make_mx(3, 64)).shape == (3, 0)
    x = torch.empty(0, 64, dtype=BF, device="cuda")
    assert ctx.block_norm_mx(ctx.make_block_norm(64, BF), x)[1].shape == (0, 64)


# ---------------------------------------------------------------------------------------------------- norms
NORM = [  # M, D, type, kind, post, gates, shift, block, alpha, pad, lead
    (1, 1, BF, "rms", True, 0, False, True, 1.0, 0, 0), (1, 4096, BF, "rms", True, 1, False, True, 1.0, 0, 0), (5, 96, HF, "layer", True, 2, True, True, 0.5, 0, 0),
    (130, 264, BF, "rms", False, 0, False, True, 1.0, 0, 0), (33, 1011, HF, "layer", True, 0, True, True, 1.0, 0, 0), (300, 1000, BF, "rms", True, 3, True, True, 0.5, 3, 1),
    (7, 2050, FF, "rms", False, 0, True, True, 1.0, 1, 1), (400, 512, FF, "layer", False, 0, False, True, 1.0, 0, 0), (2, 8200, BF, "layer", True, 1, True, True, 1.0, 0, 0),
    (310, 520, HF, "rms", False, 0, False, False, 1.0, 0, 0), (3, 32768, BF, "rms", True, 0, False, True, 1.0, 0, 0), (600, 16400, HF, "layer", False, 1, False, True, 1.0, 0, 0),
    (350, 4104, FF, "rms", True, 0, False, True, 1.0, 0, 0), (2, 20001, HF, "layer", True, 0, True, True, 1.0, 0, 0), (320, 33, BF, "layer", False, 0, False, True, 1.0, 2, 0),
    (5, 16400, FF, "rms", True, 1, True, True, 0.5, 0, 0), (4, 20001, FF, "layer", True, 0, True, True, 1.0, 0, 0), (300, 16384, FF, "rms", False, 0, False, True, 1.0, 0, 0),
    (310, 8448, BF, "rms", False, 0, False, True, 1.0, 0, 0), (300, 2048, HF, "rms", False, 0, False, True, 0.5, 0, 0), (400, 512, BF, "rms", False, 0, False, True, 1.0, 0, 0),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("M,D,dtype,kind,post,gates,shift,block,alpha,pad,lead", NORM)
def test_block_norm_mx(ctx, M, D, dtype, kind, post, gates, shift, block, alpha, pad, lead, fmt):
    mk = Maker(M * 3 + D)
    x, b = mk(M, D, dtype=dtype, scale=2.0, pad=pad, lead=lead, spread=0.5), mk(M, D, dtype=dtype, shift=0.1, pad=pad, lead=lead) if block else None
    vec = lambda on, s: mk(D, dtype=dtype, scale=0.2, shift=s, lead=lead) if on else None  # noqa: E731
    rows = -(-M // max(1, gates))
    n = {"kind": kind, "eps": 1e-5, "alpha": alpha, "post": post, "pre": True, "post_weight": vec(post, 1.0), "post_shift": vec(post and shift, 0.0),
         "pre_weight": vec(True, 1.0), "pre_shift": vec(shift, 0.0), "gate": mk(gates, D, dtype=dtype, scale=0.3, shift=0.5) if gates else None, "rows_per_gate": rows}
    layer = ctx.make_block_norm(D, dtype, **n)
    q, intact = framed_mx(ctx, M, D, fmt)
    stream, values, stats = Framed(M, D, dtype, pad, lead), Framed(M, D, dtype, pad, lead), ctx.empty(M, 4, dtype=FF)
    got, out = ctx.block_norm_mx(layer, x, b, out=q, stream=stream.t, values=values.t, stats=stats)
    assert out is q and got is stream.t
    intact(), stream.check(), values.check()
    ref.check(got, *ref.block_norm(x, b, n)["stream"], "stream")
    # the norm before its quantisation: the bound of float32 arithmetic alone (inputs that are float32 have float32's half unit at the end)
    fine = {k: v.float() if torch.is_tensor(v) else v for k, v in n.items()}
    v, err = ref.block_norm(x.float(), None if b is None else b.float(), fine)["normed"]
    read, padding, _ = mx.read(q)
    mx.accept(read.cuda(), v, err, fmt, "normed")
    assert (padding == 0).all() and torch.equal(values.t, read.cuda().to(dtype))
    plain = ctx.empty(M, 4, dtype=FF)                                # the statistics are those of the 16-bit norm: its backward pass takes them
    ctx.block_norm(layer, x, b, stats=plain)
    used = [0, 1] * (block and post) + [2, 3]
    assert torch.allclose(stats[:, used], plain[:, used], rtol=1e-5, atol=1e-5 * float(plain[:, used].abs().max()))
    again = ctx.block_norm_mx(layer, x, b, format=fmt)[1]
    assert torch.equal(mx.read(again)[0], read)
    inplace = x.clone()
    ctx.block_norm_mx(layer, inplace, b, format=fmt, stream=inplace)
    assert torch.equal(inplace, stream.t)


def test_norm_decides_borders_by_the_exact_value(ctx):
    """Rows that a float32 rounding puts on the border of two elements: the element is that of the unrounded value.  8192 x 1024 values, of which float32
    arithmetic alone misplaces a few; float64 forms the same values with an error of 2^-50."""
    mk = Maker(4)
    x, w = mk(8192, 1024, scale=2.0, spread=0.5), mk(1024, scale=0.1, shift=1.0)
    layer = ctx.make_block_norm(1024, BF, pre_weight=w)
    _, q = ctx.block_norm_mx(layer, x, format="e4m3")
    v = x.double() / (x.double().pow(2).mean(1, keepdim=True) + 1e-6).sqrt() * w.double()
    off = ctx.mx_values(q).double() != mx.quantize(v, "e4m3")
    # float32 roundings of a value, its weight and root, 2^-24 each, would cross a border 2^-4 apart (2^-3 to 2^-4 of the value) for about 2^-20 of 2^23 values: eight.
    # What is left is the error of the mean square, below 2^-26: two.
    assert int(off.sum()) <= 4


# ---------------------------------------------------------------------------------------------------- products
LINEAR = [  # M, N, K, type, act, bias, residual, pad, lead
    (1, 1, 1, BF, "none", True, True, 0, 0), (1, 4096, 512, BF, "none", True, True, 0, 0), (1, 10, 784, HF, "silu", False, False, 0, 0), (3, 257, 65, HF, "relu", True, False, 1, 1),
    (17, 1000, 1016, BF, "gelu", True, True, 8, 0), (64, 128, 4100, HF, "gelu_tanh", False, True, 0, 0), (65, 136, 72, BF, "htanh", True, True, 3, 2),
    (97, 300, 260, BF, "sigmoid", True, False, 0, 8), (129, 130, 300, HF, "none", False, True, 0, 0), (193, 520, 264, HF, "none", False, True, 0, 0),
    (257, 511, 129, BF, "gelu", True, True, 5, 3), (300, 300, 2048, BF, "silu", True, False, 0, 0), (1030, 770, 392, HF, "relu", False, False, 0, 0),
    (513, 1024, 1023, BF, "none", True, True, 1, 0), (2, 70000, 64, BF, "none", False, False, 0, 0), (16, 33, 9000, BF, "none", True, False, 0, 0),
    (1500, 24, 96, BF, "silu", True, True, 0, 0), (2900, 3000, 100, BF, "gelu", True, True, 0, 0), (2304, 2336, 520, HF, "none", False, True, 0, 0), (700, 96, 160, BF, "gelu_tanh", True, True, 0, 0),
    (4000, 40, 5000, HF, "none", True, False, 0, 0),
]


@pytest.mark.parametrize("xf,wf", PAIRS)
@pytest.mark.parametrize("M,N,K,dtype,act,bias,residual,pad,lead", LINEAR)
def test_linear(ctx, M, N, K, dtype, act, bias, residual, pad, lead, xf, wf):
    mk = Maker(M * 7 + N * 3 + K)
    x, W = ctx.mx_quantize(mk(M, K, spread=1.0), xf), ctx.mx_quantize(mk(N, K, scale=K ** -0.5), wf)
    b = mk(N, dtype=dtype, lead=lead) if bias else None
    r = mk(M, N, dtype=dtype, pad=pad, lead=lead) if residual else None
    layer = ctx.make_mx_linear(W, b, act, dtype=dtype)
    want = mx.linear(ctx.mx_values(x).double(), ctx.mx_values(W).double(), b, r, act, dtype)
    y, pre = Framed(M, N, dtype, pad, lead), Framed(M, N, FF, pad, lead)
    ctx.mx_linear(layer, x, r, out=y.t, pre=pre.t)
    ctx.device_status()
    ref.check(y.t, *want["y"], "y")
    ref.check(pre.t, *want["pre"], "pre")
    y.check(), pre.check()
    y = ctx.mx_linear(layer, x, r)
    ref.check(y, *want["y"], "y without pre")
    assert torch.equal(y, ctx.mx_linear(layer, x, r)), "the same call gives other bits"
    if r is not None:
        ref.check(ctx.mx_linear(layer, x, r, out=r), *want["y"], "y in place")
    raw = mx.linear(ctx.mx_values(x).double(), ctx.mx_values(W).double(), b, None, act, dtype)["raw"]
    for fmt in FORMATS:
        q, intact = framed_mx(ctx, M, N, fmt)
        ctx.mx_linear(layer, x, out=q)
        intact()
        v, padding, _ = mx.read(q)
        mx.accept(v.cuda(), *raw, fmt, "microscaled y")
        assert (padding == 0).all()


GATED = [  # M, N, K, type, act
    (1, 1, 1, BF, "silu"), (1, 4096, 512, BF, "silu"), (3, 257, 65, HF, "relu"), (17, 1000, 1016, BF, "gelu"), (65, 136, 72, BF, "htanh"), (97, 300, 260, BF, "sigmoid"),
    (48, 2050, 2048, HF, "gelu_tanh"), (129, 300, 128, BF, "none"), (257, 511, 129, BF, "gelu"), (1030, 770, 392, HF, "relu"), (2600, 1200, 140, BF, "silu"), (1500, 24, 96, BF, "gelu_tanh"),
]


@pytest.mark.parametrize("xf,wf", PAIRS)
@pytest.mark.parametrize("M,N,K,dtype,act", GATED)
def test_gated(ctx, M, N, K, dtype, act, xf, wf):
    mk = Maker(M * 7 + N * 3 + K)
    x, Wg, Wu = ctx.mx_quantize(mk(M, K, spread=1.0), xf), ctx.mx_quantize(mk(N, K, scale=K ** -0.5), wf), ctx.mx_quantize(mk(N, K, scale=K ** -0.5), wf)
    layer = ctx.make_mx_gated(Wg, Wu, act, dtype=dtype)
    want = mx.gated(*(ctx.mx_values(t).double() for t in (x, Wg, Wu)), act, dtype)
    h, pre = Framed(M, N, dtype, 3, 1), ctx.empty(2, M, N, dtype=FF)
    ctx.mx_gated(layer, x, out=h.t, pre=pre)
    ctx.device_status()
    h.check()
    for got, key in ((h.t, "h"), (pre[0], "g"), (pre[1], "u"), (ctx.mx_gated(layer, x), "h")):
        ref.check(got, *want[key], key)
    assert torch.equal(ctx.mx_gated(layer, x), ctx.mx_gated(layer, x)), "the same call gives other bits"
    for fmt in FORMATS:
        q, intact = framed_mx(ctx, M, N, fmt)
        ctx.mx_gated(layer, x, out=q)
        intact()
        v, padding, _ = mx.read(q)
        mx.accept(v.cuda(), *want["raw"], fmt, "microscaled h")
        assert (padding == 0).all()


def test_residual_under_kept_pre_activations(ctx):
    """More tiles than CTA pairs, so that both accumulators are read, each from its own end: every output gets its own element of the residual."""
    M, N, K = 4096, 4096, 128
    zero = ctx.mx_quantize(torch.zeros(M, K, dtype=BF, device="cuda"))
    layer, pre = ctx.make_mx_linear(zero), ctx.empty(M, N, dtype=FF)
    i, j = torch.arange(M, device="cuda")[:, None], torch.arange(N, device="cuda")[None, :]
    for r in (i % 256 + 0 * j, i // 256 + 0 * j, j % 256 + 0 * i, j // 256 + 0 * i):
        r = r.to(BF)
        assert torch.equal(ctx.mx_linear(layer, zero, r, pre=pre), r)
        assert torch.equal(ctx.mx_linear(layer, zero, r), r)


def test_scales_of_the_whole_range(ctx):
    """Rows and weights from 2^-90 to 2^90 whose products come back into range: the exponents meet in the tensor cores."""
    mk = Maker(9)
    for xf, wf in PAIRS:
        e = torch.linspace(-90, 90, 64, device="cuda").round()
        x, W = mk(64, 256, dtype=FF) * torch.exp2(e)[:, None], mk(64, 256, dtype=FF) * torch.exp2(-e)[:, None]
        q, w = ctx.mx_quantize(x, xf), ctx.mx_quantize(W, wf)
        pre = ctx.empty(64, 64, dtype=FF)
        ctx.mx_linear(ctx.make_mx_linear(w), q, pre=pre)
        want = mx.linear(ctx.mx_values(q).double(), ctx.mx_values(w).double(), None, None, "none", BF)["pre"]
        ref.check(pre.diagonal(), want[0].diagonal(), want[1].diagonal(), "pre")


@pytest.mark.parametrize("M,N,K,act", [(5, 40, 70, "gelu"), (300, 264, 136, "silu"), (64, 100, 256, "none")])
def test_straight_through_gradients(ctx, M, N, K, act):
    """The 16-bit backward pass on the represented values and kept pre-activations is the gradient of the microscaled layer at those values: against
    the formula's, and against differences of the layer itself."""
    mk = Maker(M + N)
    x, W, b, dy = mk(M, K), mk(N, K, scale=K ** -0.5), mk(N), mk(M, N)
    xv, Wv = torch.empty_like(x), torch.empty_like(W)
    q, w = ctx.mx_quantize(x, "e4m3", values=xv), ctx.mx_quantize(W, "e2m1", values=Wv)
    pre = ctx.empty(M, N, dtype=FF) if act != "none" else None
    ctx.mx_linear(ctx.make_mx_linear(w, b, act), q, pre=pre)
    back = ctx.make_linear(Wv, b, act)
    n = ctx.linear_workspace_bytes(back, xv, backward=True, dy=dy)
    ctx.set_workspace(torch.empty(max(256, n), dtype=torch.uint8, device="cuda"))
    want = ref.linear(xv, Wv, b, None, act, dy)
    grads = dict(zip(("dx", "dW", "db"), ctx.linear_backward(back, dy, xv, pre)))
    for key, t in grads.items():
        ref.check(t, *want[key], key)
    ctx.set_workspace(None)
    # differences: the same layer at weights one element apart, in its own pre-activations (exact to float32)
    i, j = 1, 3
    up = Wv.clone()
    block = up[i, j // 32 * 32:j // 32 * 32 + 32].float().abs()
    step = float(torch.exp2(mx.exponent(block.max()[None].double(), "e2m1").double()) * 0.5)
    up[i, j] += step if abs(float(up[i, j])) < 4 * step else (-step if float(up[i, j]) > 0 else step) * 4
    z = [ctx.empty(M, N, dtype=FF) for _ in range(2)]
    for t, v in zip(z, (Wv, up)):
        ctx.mx_linear(ctx.make_mx_linear(ctx.mx_quantize(v, "e2m1"), b, act), q, pre=t)
    moved = float(up[i, j].double() - Wv[i, j].double())
    slope = (z[1] - z[0])[:, i].double() / moved                     # d z / d W[i, j]: the column of x
    assert torch.allclose(slope, xv[:, j].double(), rtol=0, atol=float(2 * mx.linear(xv.double(), Wv.double(), b, None, act, BF)["pre"][1][:, i].max() / abs(moved)))


@pytest.mark.parametrize("M,N,K", [(5, 40, 70), (300, 264, 136)])
def test_straight_through_gradients_of_gated(ctx, M, N, K):
    mk = Maker(M + N)
    x, Wg, Wu, dh = mk(M, K), mk(N, K, scale=K ** -0.5), mk(N, K, scale=K ** -0.5), mk(M, N)
    xv, gv, uv = (torch.empty_like(t) for t in (x, Wg, Wu))
    q, g, u = ctx.mx_quantize(x, "e4m3", values=xv), ctx.mx_quantize(Wg, "e2m1", values=gv), ctx.mx_quantize(Wu, "e2m1", values=uv)
    pre = ctx.empty(2, M, N, dtype=FF)
    ctx.mx_gated(ctx.make_mx_gated(g, u), q, pre=pre)
    back = ctx.make_gated(gv, uv)
    ctx.set_workspace(torch.empty(max(256, ctx.gated_workspace_bytes(back, xv, backward=True)), dtype=torch.uint8, device="cuda"))
    want = ref.gated(xv, gv, uv, "silu", dh)
    for key, t in zip(("dx", "dWg", "dWu"), ctx.gated_backward(back, dh, xv, pre)):
        ref.check(t, *want[key], key)
    ctx.set_workspace(None)


def test_scales_of_rows_that_do_not_exist_may_be_anything(ctx):
    """Scale bytes are kept for 128 rows at a time.  NaN (255) in those of rows that do not exist reaches nothing, of x and of the weights, on both kernels."""
    mk = Maker(8)
    for M, N in ((3, 40), (150, 200), (700, 1050)):
        for xf, wf in PAIRS:
            x, W, U = mk(M, 200), mk(N, 200), mk(N, 200)
            got = []
            for fill in (255, 0):
                q, w, u = ctx.make_mx(M, 200, xf), ctx.make_mx(N, 200, wf), ctx.make_mx(N, 200, wf)
                for t, v in ((q, x), (w, W), (u, U)):
                    t.scales.fill_(fill)
                    ctx.mx_quantize(v, out=t)
                h = ctx.mx_gated(ctx.make_mx_gated(w, u), q, out=ctx.make_mx(M, N, "e4m3"))
                got.append((ctx.mx_linear(ctx.make_mx_linear(w), q), ctx.mx_gated(ctx.make_mx_gated(w, u), q), ctx.mx_values(h)))
            for a, b in zip(*got):
                assert a.isfinite().all() and torch.equal(a, b)


def test_offsets_beyond_32_bits(ctx):
    """More than 2^31 elements: the last rows are as they would be alone."""
    M, K = 36000, 66000
    x = torch.empty(M, K, dtype=BF, device="cuda").normal_()
    q = ctx.mx_quantize(x, "e4m3")
    out = ctx.mx_values(q, BF)
    assert torch.equal(out[-3:], mx.quantize(x[-3:].double(), "e4m3").to(BF))
    norm = ctx.make_block_norm(32768, BF)
    wide = x.view(-1)[:72000 * 32768].view(72000, 32768)
    stream, n = ctx.block_norm_mx(norm, wide, format="e4m3")
    small = ctx.block_norm_mx(norm, wide[-128:], format="e4m3")[1]            # 72000 rows: the last 64 are half a tile of scales
    assert torch.equal(ctx.mx_values(n, BF)[-64:], ctx.mx_values(small, BF)[-64:]) and torch.equal(stream[-3:], wide[-3:])
    del out, wide, stream, n
    w = ctx.mx_quantize(Maker(1)(64000, 96), "e4m3")
    q = ctx.mx_quantize(x[:, :96], "e4m3")
    y, pre = torch.empty(M, 64000, dtype=BF, device="cuda"), torch.empty(M, 64000, device="cuda")
    layer = ctx.make_mx_linear(w)
    ctx.mx_linear(layer, q, out=y, pre=pre)
    want = mx.linear(ctx.mx_values(q)[-5:].double(), ctx.mx_values(w).double(), None, None, "none", BF)
    ref.check(y[-5:], *want["y"], "y"), ref.check(pre[-5:], *want["pre"], "pre")
    del pre
    h = ctx.mx_linear(layer, q, out=ctx.make_mx(M, 64000, "e2m1"))
    v = ctx.mx_values(h, BF)
    mx.accept(v[-5:], *want["raw"], "e2m1", "microscaled y")


def test_contexts_of_two_threads(ctx):
    """A context per host thread: both kernels' one-time preparations and launches from two threads at once."""
    mk = Maker(2)
    q, big, w = ctx.mx_quantize(mk(5, 512)), ctx.mx_quantize(mk(900, 512)), ctx.mx_quantize(mk(700, 512), "e2m1")
    layer = ctx.make_mx_linear(w)
    want = ctx.mx_linear(layer, q), ctx.mx_linear(layer, big)
    torch.cuda.synchronize()
    failures = []

    def work(i):
        try:
            s = torch.cuda.Stream()
            c = binding.Context(0, s)
            with torch.cuda.stream(s):
                for _ in range(200):
                    got = c.mx_linear(layer, q), c.mx_linear(layer, big)
                s.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(got, want))
                c.device_status()
            c.close()
        except Exception as e:                    # raised in the test's own thread below
            failures.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures


def test_other_streams_and_graphs(ctx):
    """A context on a stream of its own called from another, and a captured chain of norm, gated projections, product and norm replayed on new inputs."""
    mk = Maker(12)
    D, F, M = 256, 384, 40
    x, b = mk(M, D), mk(M, D)
    side = torch.cuda.Stream()
    c = binding.Context(0, side)
    Wg, Wu, Wd, w = mk(F, D, scale=D ** -0.5), mk(F, D, scale=D ** -0.5), mk(D, F, scale=F ** -0.5), mk(D, shift=1.0, scale=0.1)

    def program(k, x, b):
        norm = k.make_block_norm(D, BF, pre_weight=w)
        up = k.make_mx_gated(k.mx_quantize(Wg, "e2m1"), k.mx_quantize(Wu, "e2m1"))
        down = k.make_mx_linear(k.mx_quantize(Wd, "e2m1"))

        def run():
            stream, n = k.block_norm_mx(norm, x, b)
            return stream, k.mx_linear(down, k.mx_gated(up, n, out=k.make_mx(M, F)), stream)
        return run

    want = [t.clone() for t in program(ctx, x, b)()]
    side.wait_stream(torch.cuda.current_stream())
    got = program(c, x, b)()                                         # called while torch's current stream is another
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    with torch.cuda.stream(side):
        run = program(c, x, b)
        run()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = run()
        for seed in (1, 2):
            x.copy_(Maker(seed)(M, D)), b.copy_(Maker(seed + 10)(M, D))
            graph.replay()
            side.synchronize()
            want = program(c, x, b)()
            side.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(out, want))
    c.device_status()
    del graph
    c.close()


@pytest.mark.parametrize("M", (4, 1024))
def test_waits_that_run_out_are_reported(ctx, M):
    """No operand arrives (the producers request nothing): both kernels end, say so, and run again afterwards."""
    mk = Maker(3)
    q, w = ctx.mx_quantize(mk(M, 512), "e4m3"), ctx.mx_quantize(mk(1024, 512), "e2m1")
    layer, glu = ctx.make_mx_linear(w), ctx.make_mx_gated(w, w)
    want = ctx.mx_linear(layer, q), ctx.mx_gated(glu, q)
    ctx.set_wait_limit_ns(20_000_000)
    ctx.debug_drop_loads(True)
    for call in (lambda: ctx.mx_linear(layer, q), lambda: ctx.mx_gated(glu, q), lambda: ctx.mx_gated(glu, q, out=ctx.make_mx(M, 1024))):
        call()
        with pytest.raises(binding.BnnError):
            ctx.device_status()
    ctx.debug_drop_loads(False)
    ctx.set_wait_limit_ns(2_000_000_000)
    assert torch.equal(ctx.mx_linear(layer, q), want[0]) and torch.equal(ctx.mx_gated(glu, q), want[1])
    ctx.device_status()
