"""Edges of the real-valued operators on the GPU."""
import threading

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


def normal(seed, *shape, dtype=BF, scale=1.0, shift=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(*shape, device="cuda").normal_(shift, scale, generator=g).to(dtype)


@pytest.mark.parametrize("M,N,K", [(64, 1011, 512), (512, 1010, 1024), (3, 9, 8)])
@pytest.mark.parametrize("bias", (True, False), ids=("bias", "plain"))
def test_linear_backward_in_the_workspace_asked_for(ctx, M, N, K, bias):
    """x and W in whole 16-byte groups, contiguous dy not: a layer without activation copies dy."""
    x, W, dy = normal(1, M, K), normal(2, N, K, scale=K ** -0.5), normal(3, M, N)
    b = normal(4, N) if bias else None
    layer = ctx.make_linear(W, b)
    n = ctx.linear_workspace_bytes(layer, x, backward=True)
    ws = torch.full((n + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    ctx.set_workspace(ws[:n] if n else None)
    want = ref.linear(x, W, b, None, "none", dy)
    for key, t in zip(("dx", "dW", "db"), ctx.linear_backward(layer, dy, x)):
        if t is not None:
            ref.check(t, *want[key], key)
    ctx.device_status()
    assert (ws[n:] == 0x7F).all(), "written beyond the workspace"
    ctx.set_workspace(None)


def test_contexts_of_two_threads_at_different_widths():
    """A context per host thread is allowed: what one thread's launches need must not depend on the other's.  Both widths run the same
    kernel with different amounts of shared memory."""
    widths, failures, results = (2048, 4096), [], {}

    def steps(D, start):
        try:
            stream = torch.cuda.Stream()
            c = binding.Context(0, stream)
            with torch.cuda.stream(stream):
                x, b, ds, dn, w = (normal(k, 4, D) for k in range(5))
                layer = c.make_block_norm(D, BF, kind="layer", post=True, pre_weight=w[0])
                ws = torch.empty(c.block_norm_workspace_bytes(layer, 4), dtype=torch.uint8, device="cuda")
                c.set_workspace(ws)
                stats = c.empty(4, 4, dtype=FF)
                c.block_norm(layer, x, b, stats=stats)
                start.wait()
                for _ in range(3000):
                    results[D] = c.block_norm_backward(layer, ds, dn, x, b, stats)["dblock"]
            stream.synchronize()
            c.close()
        except Exception as e:                    # raised in the test's own thread below
            failures.append(e)

    build.build()
    start = threading.Barrier(len(widths), timeout=60)
    threads = [threading.Thread(target=steps, args=(D, start)) for D in widths]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures, failures
    for D in widths:
        x, b, ds, dn, w = (normal(k, 4, D) for k in range(5))
        par = {"kind": "layer", "eps": 1e-6, "alpha": 1.0, "post": True, "pre": True, "pre_weight": w[0]}
        ref.check(results[D], *ref.block_norm(x, b, par, ds, dn)["dblock"], "dblock")


@pytest.mark.parametrize("M,N", [(0, 8), (4, 0)])
@pytest.mark.parametrize("act", ("none", "silu"))
def test_empty_backward_with_every_pointer_given(ctx, M, N, act):
    """The C entry points with operands off the 16-byte rule and no workspace, which is what the size functions ask for."""
    K, L = 9, binding.lib()
    x, W, dy, room = normal(1, 4, K), normal(2, 8, K), normal(3, 4, 8), normal(4, 8, 8, dtype=FF)
    b = normal(5, 8)
    code = binding.ACTIVATIONS[act]
    lin = binding.LinearDesc(binding.BNN_BF16, code, K, N, W.data_ptr(), K, b.data_ptr())
    glu = binding.GatedDesc(binding.BNN_BF16, code, K, N, W.data_ptr(), K, W.data_ptr(), K)
    assert L.bnn_linear_workspace_bytes(lin, M, 1, 0) == L.bnn_gated_workspace_bytes(glu, M, 1, 0) == 0
    ctx.set_workspace(None)
    dx, dW, dU, db = (torch.full(s, 5.0, dtype=BF, device="cuda") for s in ((4, K), (8, K), (8, K), (8,)))
    for pre in (None, room.data_ptr()):
        for t in (dx, dW, dU, db):
            t.fill_(5.0)
        assert L.bnn_linear_backward(ctx._h, lin, dy.data_ptr(), 8, x.data_ptr(), K, M, pre, 8, dx.data_ptr(), K, dW.data_ptr(), K, db.data_ptr()) == 0
        assert (dx[:M] == 0).all() and (dx[M:] == 5).all() and (dW[:N] == 0).all() and (dW[N:] == 5).all() and (db[:N] == 0).all() and (db[N:] == 5).all()
        dx.fill_(5.0), dW.fill_(5.0)
        assert L.bnn_gated_backward(ctx._h, glu, dy.data_ptr(), 8, x.data_ptr(), K, M, pre, 8, dx.data_ptr(), K, dW.data_ptr(), K, dU.data_ptr(), K) == 0
        assert (dx[:M] == 0).all() and (dx[M:] == 5).all() and (dW[:N] == 0).all() and (dU[:N] == 0).all() and (dU[N:] == 5).all()
    ctx.device_status()


@pytest.mark.parametrize("rows_per_gate", (9, 0x7fffffff, (1 << 63) - 1))
def test_one_gate_row_that_covers_more_rows_than_there_are(ctx, rows_per_gate):
    M, D = 9, 72
    x, b, ds, dn, gate = normal(1, M, D), normal(2, M, D), normal(3, M, D), normal(4, M, D), normal(5, 1, D)
    layer = ctx.make_block_norm(D, BF, post=True, gate=gate, rows_per_gate=rows_per_gate)
    ws = torch.empty(ctx.block_norm_workspace_bytes(layer, M), dtype=torch.uint8, device="cuda")
    ctx.set_workspace(ws)
    par = {"kind": "rms", "eps": 1e-6, "alpha": 1.0, "post": True, "pre": True, "gate": gate, "rows_per_gate": M}
    want = ref.block_norm(x, b, par, ds, dn)
    stats = ctx.empty(M, 4, dtype=FF)
    for key, t in zip(("stream", "normed"), ctx.block_norm(layer, x, b, stats=stats)):
        ref.check(t, *want[key], key)
    for key, t in ctx.block_norm_backward(layer, ds, dn, x, b, stats).items():
        if t is not None:
            ref.check(t, *want[key], key)
    ctx.set_workspace(None)


@pytest.mark.parametrize("M,N,K", [(1, 300, 4096), (130, 1000, 64), (700, 8192, 512)], ids=("split", "few", "tiles in turn"))
def test_waits_that_run_out_in_every_epilogue(M, N, K):
    """Nothing is loaded, so that every warp of an epilogue gives up, as one: statuses, and right results afterwards."""
    c = binding.Context(0)
    x, W, U, dy = normal(1, M, K), normal(2, N, K, scale=K ** -0.5), normal(3, N, K, scale=K ** -0.5), normal(4, M, N)
    layer, glu, pre = c.make_linear(W, None, "silu"), c.make_gated(W, U), c.empty(2, M, N, dtype=FF)
    ws = torch.empty(max(c.linear_workspace_bytes(layer, x, backward=True), c.gated_workspace_bytes(glu, x, backward=True)), dtype=torch.uint8, device="cuda")
    c.set_workspace(ws)
    c.set_wait_limit_ns(5_000_000)
    for call in (lambda: c.linear(layer, x, pre=pre[0]), lambda: c.gated(glu, x, pre=pre), lambda: c.linear_backward(layer, dy, x),
                 lambda: c.gated_backward(glu, dy, x)):
        c.debug_drop_loads(True)
        call()
        with pytest.raises(binding.BnnError) as e:
            c.device_status()
        assert e.value.status == -5
        c.debug_drop_loads(False)
    ref.check(c.linear(layer, x), *ref.linear(x, W, None, None, "silu")["y"], "y after failures")
    ref.check(c.gated(glu, x), *ref.gated(x, W, U, "silu")["h"], "h after failures")
    c.device_status()
    c.set_workspace(None)
    c.close()


@pytest.mark.parametrize("M,N,K", [(1, 300, 4096), (130, 1000, 64), (700, 1000, 128), (700, 8192, 1024)], ids=("split", "few", "pairs", "tiles in turn"))
def test_waits_that_run_out_with_copies_in_flight(M, N, K):
    """The shortest limit that can be set, with the loads on: waits may give up at any point while copies and products are under way.  Either
    a status or a right result, nothing beyond the output written, and right results afterwards."""
    c = binding.Context(0)
    x, W, U, dy = normal(1, M, K), normal(2, N, K, scale=K ** -0.5), normal(3, N, K, scale=K ** -0.5), normal(4, M, N)
    layer, glu = c.make_linear(W, None, "silu"), c.make_gated(W, U)
    n = max(c.linear_workspace_bytes(layer, x, backward=True), c.gated_workspace_bytes(glu, x, backward=True))
    ws = torch.full((n + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    c.set_workspace(ws[:n])
    want = {"y": ref.linear(x, W, None, None, "silu")["y"], "h": ref.gated(x, W, U, "silu")["h"]}
    room = torch.full((M + 2, N), 5.0, dtype=BF, device="cuda")
    for key, call in (("y", lambda out: c.linear(layer, x, out=out)), ("h", lambda out: c.gated(glu, x, out=out)),
                      (None, lambda out: c.linear_backward(layer, dy, x)), (None, lambda out: c.gated_backward(glu, dy, x))):
        for _ in range(4):
            c.set_wait_limit_ns(1)
            call(room[1:-1])
            try:
                c.device_status()
                if key:
                    ref.check(room[1:-1], *want[key], key)
            except binding.BnnError as e:
                assert e.status == -5
            assert (room[0] == 5).all() and (room[-1] == 5).all() and (ws[n:] == 0x7F).all()
        c.set_wait_limit_ns(2_000_000_000)
        call(room[1:-1])
        c.device_status()
        if key:
            ref.check(room[1:-1], *want[key], key + " afterwards")
    c.set_workspace(None)
    c.close()


# act(z) and act'(z) in 64 bits, each without a difference that cancels far out, the lowest z whose results are normal numbers of bfloat16, and
# how far the exponent may be off: |exponent| times a few 2^-24.
def phi64(z):
    return 0.5 * torch.special.erfc(-z / 2 ** 0.5), torch.exp(-0.5 * z * z) / (2 * torch.pi) ** 0.5


def gelu64(z):
    cdf, density = phi64(z)
    return z * cdf, cdf + z * density, cdf + z.abs() * density


def gelu_tanh_exponent(z):
    return (8 / torch.pi) ** 0.5 * (z + 0.044715 * z ** 3)


def gelu_tanh64(z):
    w = gelu_tanh_exponent(z)
    s, steep = torch.sigmoid(w), torch.sigmoid(-w) * (8 / torch.pi) ** 0.5 * (1 + 3 * 0.044715 * z * z)
    return z * s, s * (1 + z * steep), s * (1 + z.abs() * steep)


def silu64(z):
    s = torch.sigmoid(z)
    return z * s, s * (1 + z * torch.sigmoid(-z)), s * (1 + z.abs())


def sigmoid64(z):
    s = torch.sigmoid(z)
    return s, s * torch.sigmoid(-z), s


TAILS = {"gelu": (gelu64, -12.5, lambda z: 0.5 * z * z), "gelu_tanh": (gelu_tanh64, -9.5, lambda z: gelu_tanh_exponent(z).abs()),
         "silu": (silu64, -80.0, torch.abs), "sigmoid": (sigmoid64, -80.0, torch.abs)}


@pytest.mark.parametrize("dtype", (BF, HF))
@pytest.mark.parametrize("act", TAILS)
def test_activation_tails_are_relatively_exact(ctx, act, dtype):
    """z = x (one input, weight 1), from far out to 4: values and slopes to a unit of the result's type and what a float32 evaluation may
    lose of the magnitude form, wherever z is."""
    form, low, exponent = TAILS[act]
    x = torch.linspace(low, 4.0, 4096, device="cuda").to(dtype)[:, None]
    layer = ctx.make_linear(torch.ones(1, 1, dtype=dtype, device="cuda"), None, act)
    ws = torch.empty(max(256, ctx.linear_workspace_bytes(layer, x, backward=True)), dtype=torch.uint8, device="cuda")
    ctx.set_workspace(ws)
    z = x.double()
    value, slope, magnitude = form(z)
    rel = 2.0 ** -18 + 2.0 ** -21 * exponent(z)
    unit, tiny = ref.UNIT[dtype], {BF: 2.0 ** -133, HF: 2.0 ** -25}[dtype]
    pre = ctx.empty(4096, 1, dtype=FF)
    ref.check(ctx.linear(layer, x, pre=pre), value, (unit + rel) * value.abs() + tiny, "value")
    # h = act(g) u with u = 1, and its product's u goes through untouched
    one = torch.ones(1, 2, dtype=dtype, device="cuda")
    glu, pair = ctx.make_gated(one * torch.tensor([1, 0], device="cuda"), one * torch.tensor([0, 1], device="cuda"), act), torch.cat((x, torch.ones_like(x)), 1)
    ws2 = torch.empty(ctx.gated_workspace_bytes(glu, pair, backward=True), dtype=torch.uint8, device="cuda")
    ctx.set_workspace(ws2)
    ref.check(ctx.gated(glu, pair), value, (unit + rel) * value.abs() + tiny, "gated value")
    dh = torch.ones_like(x)
    ref.check(ctx.gated_backward(glu, dh, pair)[0], torch.cat((slope, value), 1),
              torch.cat((unit * slope.abs() + rel * magnitude, (unit + rel) * value.abs()), 1) + 2 * tiny, "gated slope and value")
    ctx.set_workspace(ws)
    for kept in (pre, None):
        dx = ctx.linear_backward(layer, dh, x, kept)[0]       # the rounded dz itself
        ref.check(dx, slope, unit * slope.abs() + rel * magnitude + 2 * tiny, "slope")
    ctx.device_status()
    ctx.set_workspace(None)


def padded(t, pad):
    """The same values in rows with `pad` more columns of NaN between them."""
    wide = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


# Several tiles a pair (a GPU has 74 pairs, a tile 256 x 256 outputs, of gated projections 256 x 128): the ring of stages runs on from tile to tile and the
# two accumulators alternate.  Sums on both sides of the 32 K steps where the number of epilogue warps changes.
@pytest.mark.parametrize("M,N,K,dtype,act,pad", [(2560, 2560, 520, HF, "silu", 0), (2560, 2560, 2056, BF, "gelu", 0), (2600, 2500, 520, BF, "none", 3)])
def test_linear_of_many_tiles(ctx, M, N, K, dtype, act, pad):
    x, W, b = normal(1, M, K, dtype=dtype), normal(2, N, K, dtype=dtype, scale=K ** -0.5), normal(3, N, dtype=dtype)
    r, dy = (padded(normal(k, M, N, dtype=dtype), pad) for k in (4, 5))
    layer = ctx.make_linear(W, b, act)
    n = ctx.linear_workspace_bytes(layer, x, backward=True, dy=dy)
    ws = torch.full((n + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    ctx.set_workspace(ws[:n])
    want, pre = ref.linear(x, W, b, r, act, dy), ctx.empty(M, N, dtype=FF)
    ref.check(ctx.linear(layer, x, r), *want["y"], "y")
    ref.check(ctx.linear(layer, x, r, pre=pre), *want["y"], "y with pre")
    ref.check(pre, *want["pre"], "pre")
    got = [ctx.linear_backward(layer, dy, x, kept) for kept in (pre, None)]
    ctx.device_status()
    for grads in got:
        for key, t in zip(("dx", "dW", "db"), grads):
            ref.check(t, *want[key], key)
    assert all(torch.equal(p, q) for p, q in zip(got[0][:2], got[1][:2])), "kept and recomputed pre-activations give other products"
    assert (ws[n:] == 0x7F).all(), "written beyond the workspace"
    ctx.set_workspace(None)


@pytest.mark.parametrize("M,N,K,dtype,act", [(2560, 2000, 520, BF, "silu"), (2560, 2000, 2056, HF, "gelu_tanh")])
def test_gated_of_many_tiles(ctx, M, N, K, dtype, act):
    x, dh = normal(1, M, K, dtype=dtype), normal(4, M, N, dtype=dtype)
    Wg, Wu = (normal(k, N, K, dtype=dtype, scale=K ** -0.5) for k in (2, 3))
    layer = ctx.make_gated(Wg, Wu, act)
    n = ctx.gated_workspace_bytes(layer, x, backward=True)
    ws = torch.full((n + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    ctx.set_workspace(ws[:n])
    want, pre = ref.gated(x, Wg, Wu, act, dh), ctx.empty(2, M, N, dtype=FF)
    ref.check(ctx.gated(layer, x), *want["h"], "h")
    ref.check(ctx.gated(layer, x, pre=pre), *want["h"], "h with pre")
    ref.check(pre[0], *want["g"], "g"), ref.check(pre[1], *want["u"], "u")
    for kept in (pre, None):
        for key, t in zip(("dx", "dWg", "dWu"), ctx.gated_backward(layer, dh, x, kept)):
            ref.check(t, *want[key], key)
    ctx.device_status()
    assert (ws[n:] == 0x7F).all(), "written beyond the workspace"
    ctx.set_workspace(None)
